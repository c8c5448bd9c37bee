"""CPU: a Kv4Cache whose tensors are replaced or copied after its first use: what goes to the library are the tensors
that it has, and they are checked as the constructor's are."""
import copy
import pickle

import pytest
import torch

from paper_2606_15682_amd import reqat

ARRAYS = ("k_codes", "k_scales", "v_codes", "v_scales")


def used(**kw):
    c = reqat.Kv4Cache(3, 16, 2, 64, k_scale=0.5, v_scale=0.25, k_shift=torch.arange(128.0), device="cpu", **kw)
    assert c.struct.k_codes == c.k_codes.data_ptr()          # as a first call takes it
    return c


def agrees(c):
    s = c.struct
    for name in ARRAYS:
        assert getattr(s, name) == getattr(c, name).data_ptr(), name
    assert s.k_tensor_scale == c.k_scale.data_ptr() and s.v_tensor_scale == c.v_scale.data_ptr()
    assert s.k_shift == (None if c.k_shift is None else c.k_shift.data_ptr())


def test_assigned_tensors_are_the_ones_used():
    c = used()
    c.k_shift = torch.ones(128)
    agrees(c)
    c.k_shift = None
    agrees(c)
    c.k_scale = torch.tensor([2.0])
    c.v_scale = 0.125
    agrees(c)
    assert c.v_scale.dtype == torch.float32 and float(c.v_scale) == 0.125
    for name in ARRAYS:
        setattr(c, name, torch.ones_like(getattr(c, name)))
        agrees(c)


def test_assigned_tensors_are_checked():
    c = used()
    for name, bad in [("k_shift", torch.zeros(127)), ("k_shift", torch.zeros(128, dtype=torch.float64)),
                      ("k_scale", 0.0), ("v_scale", float("nan")), ("k_scale", torch.ones(1, dtype=torch.float64))] + \
                     [(n, torch.zeros(7, dtype=torch.uint8)) for n in ARRAYS] + \
                     [(n, torch.zeros(getattr(c, n).numel(), dtype=torch.int8)) for n in ARRAYS] + \
                     [(n, torch.zeros(2 * getattr(c, n).numel(), dtype=torch.uint8)[::2]) for n in ARRAYS]:
        before = getattr(c, name)
        with pytest.raises((TypeError, ValueError)):
            setattr(c, name, bad)
        assert getattr(c, name) is before
    agrees(c)


@pytest.mark.parametrize("name", ["num_pages", "page_size", "kv_heads", "head_dim", "width", "device"])
def test_sizes_stay(name):
    c = used()
    with pytest.raises(AttributeError):
        setattr(c, name, getattr(c, name))


def test_copies_have_their_own_tensors():
    c = used()
    c.k_codes.fill_(7)
    for d in (copy.deepcopy(c), pickle.loads(pickle.dumps(c))):
        agrees(d)
        assert d.k_codes.data_ptr() != c.k_codes.data_ptr() and torch.equal(d.k_codes, c.k_codes)
        assert (d.num_pages, d.page_size, d.kv_heads, d.head_dim) == (3, 16, 2, 64)
    d = copy.copy(c)
    agrees(d)
    d.k_shift = torch.full((128,), 3.0)
    agrees(d)
    agrees(c)
    assert c.k_shift.data_ptr() != d.k_shift.data_ptr()


@pytest.mark.parametrize("g", [1e-50, 1e39, 0.0, -1.0, float("inf"), float("nan")])
def test_scales_are_positive_finite_fp32_numbers(g):
    """A number that FP32 holds as zero or infinity is no scale either."""
    for name in ("k_scale", "v_scale"):
        with pytest.raises(ValueError):
            reqat.Kv4Cache(1, 16, 1, 64, device="cpu", **{name: g})
    assert float(reqat.Kv4Cache(1, 16, 1, 64, device="cpu", k_scale=1e-45).k_scale) > 0.0
