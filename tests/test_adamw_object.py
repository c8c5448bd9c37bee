"""AdamW's host side on CPU tensors, with the C calls recorded instead of made: what a step hands over."""
import copy

import pytest
import torch

from paper_2606_15682_amd import reqat

WORDS = ("p", "g", "m", "v", "m_scale", "v_scale", "copy", "n")


@pytest.fixture
def calls(monkeypatch):
    """The calls made: (name of the C function, its arguments, the descriptors as dicts where it takes some)."""
    made = []

    def record(fn, device, *args):
        words = None
        if fn is reqat.reqat_adamw_step:
            words = [dict(zip(WORDS, args[0][8 * i:8 * i + 8])) for i in range(args[1])]
        made.append((fn.__name__, args, words))

    monkeypatch.setattr(reqat, "_call", record)
    monkeypatch.setattr(reqat, "_require_cuda", lambda *a: None)
    return made


def _params():
    return [torch.ones(10), torch.ones(3, 4), torch.ones(7)]


def _grads():
    return [torch.ones(10), torch.ones(3, 4), torch.ones(7)]


def _steps(calls):
    return [(args, words) for name, args, words in calls if name == "reqat_adamw_step"]


@pytest.mark.parametrize("bits", [8, 32])
def test_copies_taken_away_and_given(calls, bits):
    """Without copies no address of an earlier step's stays in the descriptors; given ones are the ones handed over."""
    p, g = _params(), _grads()
    copies = [torch.empty(10, dtype=torch.bfloat16), None, torch.empty(7, dtype=torch.bfloat16)]
    opt = reqat.AdamW(p, 1e-3, state_bits=bits, copies=copies)
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [copies[0].data_ptr(), 0, copies[2].data_ptr()]
    opt.copies = None
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [0, 0, 0]
    opt.copies = [None, torch.empty(3, 4, dtype=torch.bfloat16), None]
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [0, opt.copies[1].data_ptr(), 0]
    opt.copies = [None, None, None]
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [0, 0, 0]
    for wrong in ([None, None], [None] * 4):
        opt.copies = wrong
        with pytest.raises(ValueError):
            opt.step(g)
    opt.copies = None
    opt.step(g)
    assert opt.steps == 5 and len(_steps(calls)) == 5
    for x, w in zip(p, _steps(calls)[-1][1]):
        assert w["p"] == x.data_ptr() and w["n"] == x.numel()
