"""GPU: layer norm and root-mean-square norm, forward and backward, against their formulas in 64 bits."""
import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32

# columns around the borders between the groups of 64, 256 and 1024 threads, odd ones, one
COLS = [1, 2, 7, 8, 9, 63, 511, 512, 513, 1024, 1536, 2047, 2049, 3584, 5120, 8193, 8960]


def _inputs(M, K, dtype, wdtype, seed=0, pad=0):
    g = torch.Generator().manual_seed(7919 * M + K + seed)
    make = lambda s: torch.randn(s, generator=g)
    x = (make((M, K + pad)) * (1 + 4 * (torch.arange(K + pad) % 97 == 0)) + 0.7 * make((M, 1))).to(dtype).to(DEV)[:, :K]
    dy = (make((M, K + pad)) * 0.1).to(dtype).to(DEV)[:, :K]
    w, b = ((1 + 0.2 * make(K)).to(wdtype).to(DEV), (0.1 * make(K)).to(wdtype).to(DEV))
    return x, dy, w, b


def _check_forward(x, w, b, center, y, stats, eps=1e-6):
    ey, es = ref.norm(x, w, b, eps, center)
    K = x.shape[1]
    X = x.double().cpu()
    deep = K / 1024 + 16                                   # additions in a row, and of the tree
    mean_tol = ref.EPS32 * deep * X.abs().mean(1) * 2
    assert torch.all((stats[:, 0].double().cpu() - es[:, 0]).abs() <= mean_tol * (1 if center else 0))
    # the mean's error shifts the variance by its square; every square carries 3 half steps, the sum `deep`, the root 3
    spread = 1 / es[:, 1]
    rel = ref.EPS32 * (2 * deep + 12) + (mean_tol / spread) ** 2 + 2 * ref.EPS32 * X.abs().amax(1) / spread
    assert torch.all((stats[:, 1].double().cpu() - es[:, 1]).abs() <= es[:, 1] * rel)
    h = (X - es[:, :1]).abs() * es[:, 1:] * w.double().cpu().abs()
    room = h * (rel + 8 * ref.EPS32)[:, None] + (mean_tol * es[:, 1])[:, None] * w.double().cpu().abs() \
        + ref.EPS32 * (X.abs() * es[:, 1:] * w.double().cpu().abs() + 2 * ey.abs())
    assert torch.all((y.double().cpu() - ey).abs() <= 1.01 * ref.half_step(x.dtype) * ey.abs() + room + 1e-37)


def _check_backward(dy, x, w, stats, center, dx, dw, db, bias):
    edx, edw, edb = ref.norm_backward(dy, x, w, stats, center)
    M, K = x.shape
    X, D, W, S = x.double().cpu(), dy.double().cpu(), w.double().cpu(), stats.double().cpu()
    mu = S[:, :1] if center else torch.zeros((M, 1), dtype=torch.float64)
    h = ((X - mu) * S[:, 1:]).abs()
    g = (D * W).abs()
    deep = K / 1024 + 24
    size = S[:, 1:] * (g + g.mean(1, keepdim=True) + h * (g * h).mean(1, keepdim=True))
    shift = ref.EPS32 * (X.abs() + mu.abs()) * S[:, 1:]    # x - mu rounds at the size of x
    room = size * ref.EPS32 * (deep + 16) + S[:, 1:] * ((g * h).mean(1, keepdim=True) * shift + h * (g * shift).mean(1, keepdim=True))
    assert torch.all((dx.double().cpu() - edx).abs() <= 1.01 * ref.half_step(x.dtype) * edx.abs() + room + 1e-37)
    rows = M / 256 + 64                                    # of a group, and of the join
    tol = ref.EPS32 * (rows + 4) * (D.abs() * h).sum(0) + (D.abs() * shift).sum(0)
    assert torch.all((dw.double().cpu() - edw).abs() <= tol + 1.01 * ref.half_step(w.dtype) * edw.abs() + 1e-37)
    if bias:
        tol = ref.EPS32 * rows * D.abs().sum(0)
        assert torch.all((db.double().cpu() - edb).abs() <= tol + 1.01 * ref.half_step(w.dtype) * edb.abs() + 1e-37)
    else:
        assert db is None


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype,wdtype", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("K", COLS)
def test_norm(K, dtype, wdtype, center):
    print("norm", K, dtype, wdtype, center, flush=True)
    for M in (1, 5, 67):
        x, dy, w, b = _inputs(M, K, dtype, wdtype)
        bias = M != 5
        y, stats = reqat.layer_norm(x, w, b if bias else None, center=center)
        _check_forward(x, w, b if bias else None, center, y, stats)
        dx, dw, db = reqat.layer_norm_backward(dy, x, w, stats, center=center, bias=bias)
        _check_backward(dy, x, w, stats, center, dx, dw, db, bias)


@pytest.mark.parametrize("K,dtype", [(16385, BF), (27648, BF), (32768, BF), (9000, F32), (16384, F32), (20001, F32),
                                     (27648, F32), (32768, F32)])
def test_wide_rows(K, dtype):
    x, dy, w, b = _inputs(3, K, dtype, F32)
    y, stats = reqat.layer_norm(x, w, b)
    _check_forward(x, w, b, True, y, stats)
    dx, dw, db = reqat.layer_norm_backward(dy, x, w, stats, bias=True)
    _check_backward(dy, x, w, stats, True, dx, dw, db, True)


@pytest.mark.parametrize("M,K", [(3001, 64), (2500, 1536), (1111, 5120), (600, 9000)])
def test_more_rows_than_groups(M, K):
    x, dy, w, b = _inputs(M, K, BF, F32)
    y, stats = reqat.layer_norm(x, w, b)
    _check_forward(x, w, b, True, y, stats)
    dx, dw, db = reqat.layer_norm_backward(dy, x, w, stats, bias=True)
    _check_backward(dy, x, w, stats, True, dx, dw, db, True)
    again = reqat.layer_norm_backward(dy, x, w, stats, bias=True)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("pad", [1, 5, 8])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_and_in_place(pad, dtype):
    x, dy, w, b = _inputs(41, 1003, dtype, F32, pad=pad)
    y, stats = reqat.layer_norm(x, w, b)
    _check_forward(x, w, b, True, y, stats)
    wide = torch.full((41, 1009), 3.0, dtype=dtype, device=DEV)
    out, s2 = reqat.layer_norm(x, w, b, out=wide[:, 3:1006])
    assert torch.equal(out, y) and torch.equal(s2, stats)
    assert torch.all(wide[:, :3] == 3.0) and torch.all(wide[:, 1006:] == 3.0)
    dx, dw, db = reqat.layer_norm_backward(dy, x, w, stats, bias=True)
    for target in ("dy", "x"):
        a, c = dy.clone(), x.clone()
        got = reqat.layer_norm_backward(a, c, w, stats, bias=True, out=a if target == "dy" else c)
        assert all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))
    z = x.clone()
    assert torch.equal(reqat.layer_norm(z, w, b, out=z)[0], y)


@pytest.mark.parametrize("K,dtype", [(20000, BF), (20001, BF), (9001, F32), (20000, F32)])
def test_wide_rows_in_place(K, dtype):
    x, dy, w, b = _inputs(7, K, dtype, F32)
    stats = reqat.layer_norm(x, w, b)[1]
    want = reqat.layer_norm_backward(dy, x, w, stats, bias=True)
    for target in ("dy", "x"):
        a, c = dy.clone(), x.clone()
        got = reqat.layer_norm_backward(a, c, w, stats, bias=True, out=a if target == "dy" else c)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_constant_and_far_rows():
    """A constant row has variance 0; far means do not cost the variance its digits, for the mean is taken off first."""
    for center in (True, False):
        x = torch.full((4, 1000), 3.0, dtype=F32, device=DEV)
        x[1] = 0.0
        x[2] = 1000.0 + torch.arange(1000, device=DEV) % 2
        x[3] = 2.0 ** 50
        w = torch.ones(1000, device=DEV)
        y, stats = reqat.layer_norm(x, w, eps=1e-5, center=center)
        _check_forward(x, w, None, center, y, stats, eps=1e-5)


def test_bad_rows_stay_their_own():
    x, dy, w, b = _inputs(9, 700, F32, F32)
    y, stats = reqat.layer_norm(x, w, b)
    x[4, 3], x[6, 699] = float("nan"), float("inf")
    y2, stats2 = reqat.layer_norm(x, w, b)
    good = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(y2[good], y[good]) and torch.isnan(y2[4]).all() and torch.isnan(stats2[[4, 6], 1]).all()
    assert not torch.isfinite(y2[6]).all()


def test_no_rows():
    w = torch.ones(77, device=DEV)
    x = torch.empty((0, 77), device=DEV)
    y, stats = reqat.layer_norm(x, w)
    assert y.shape == (0, 77) and stats.shape == (0, 2)
    dx, dw, db = reqat.layer_norm_backward(x, x, w, stats, bias=True)
    assert dx.shape == (0, 77) and not dw.any() and not db.any()


def test_against_differences_and_autograd():
    """Central differences of sum(y c): third derivatives of order one, times h^2; FP32 rounding of y over h."""
    x, c, w, b = _inputs(3, 11, F32, F32)
    c = c.contiguous()
    for center in (True, False):
        leaves = [t.clone().requires_grad_() for t in (x.contiguous(), w, b)]
        (reqat.LayerNorm.apply(*leaves, 1e-3, center) * c).sum().backward()
        h = 2.0 ** -6
        for k, leaf in enumerate(leaves):
            flat = leaf.grad.flatten()
            for j in range(flat.numel()):
                f = []
                for sign in (1, -1):
                    args = [t.detach().clone() for t in leaves]
                    args[k].view(-1)[j] += sign * h
                    f.append(float((reqat.layer_norm(*args, 1e-3, center)[0].double() * c).sum()))
                assert abs((f[0] - f[1]) / (2 * h) - float(flat[j])) <= 1e-3
    leaves = [t.clone().requires_grad_() for t in (x.contiguous(), w)]
    reqat.LayerNorm.apply(*leaves).sum().backward()        # an expanded gradient
    assert leaves[0].grad.shape == x.shape and leaves[1].grad.shape == w.shape
