"""GPU: every form of the norm kernels against 64 bits: each group size with every number of vectors a thread, more rows than
workgroups, weights' gradients by columns over parts of many rows, in place, both types."""
import pytest
import torch

from paper_2606_15682_amd import reqat

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24                                            # half a step of FP32, relative


def _inputs(M, K, dtype, wdtype, pad):
    g = torch.Generator(device=DEV).manual_seed(7919 * M + K)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)
    x = (rand(M, K + pad) * (1 + 4 * (torch.arange(K + pad, device=DEV) % 97 == 0)) + 0.7 * rand(M, 1)).to(dtype)[:, :K]
    dy = (0.1 * rand(M, K + pad)).to(dtype)[:, :K]
    return x, dy, (1 + 0.2 * rand(K)).to(wdtype), (0.1 * rand(K)).to(wdtype)


def _half(dtype):
    return 1.01 * torch.finfo(dtype).eps / 2


def _check_forward(x, w, b, center, y, stats):
    X, W = x.double(), w.double()
    K = x.shape[1]
    mu = X.mean(1, keepdim=True) if center else X.new_zeros(X.shape[0], 1)
    rstd = 1 / torch.sqrt(((X - mu) ** 2).mean(1, keepdim=True) + 1e-6)
    want = (X - mu) * rstd * W
    want = want if b is None else want + b.double()
    # sums: up to 64 elements one after the other in a thread, six steps in a wave, up to 16 waves
    deep = 64 + 6 + 16
    d_mu = E * (deep + 2) * X.abs().mean(1, keepdim=True) * (1 if center else 0)
    assert torch.all((stats[:, :1].double() - mu).abs() <= d_mu)
    # every square: 3 half steps, and x - mu rounds at x's size; the root, the quotient and the mean 4
    rel = E * (deep + 8 + 2 * (X.abs() * (X - mu).abs()).mean(1, keepdim=True) * rstd ** 2) + (d_mu * rstd) ** 2
    assert torch.all((stats[:, 1:].double() - rstd).abs() <= rstd * rel)
    room = ((X - mu).abs() * (rel + 4 * E) + d_mu + E * X.abs()) * rstd * W.abs() + 2 * E * want.abs()
    assert torch.all((y.double() - want).abs() <= _half(x.dtype) * want.abs() + room + 1e-37)


def _check_backward(dy, x, w, stats, center, dx, dw, db):
    X, D, W, S = x.double(), dy.double(), w.double(), stats.double()
    M = x.shape[0]
    mu = S[:, :1] if center else S.new_zeros(M, 1)
    h, g = (X - mu) * S[:, 1:], D * W
    mg, mgh = g.mean(1, keepdim=True) * (1 if center else 0), (g * h).mean(1, keepdim=True)
    want = (g - mg - h * mgh) * S[:, 1:]
    d_h = E * ((X.abs() + mu.abs()) * S[:, 1:] + 2 * h.abs())      # x - mu rounds at its terms' size
    deep = 64 + 6 + 16
    size = g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)
    room = S[:, 1:] * (size * E * (deep + 12) + d_h * mgh.abs() + h.abs() * (g.abs() * d_h).mean(1, keepdim=True))
    assert torch.all((dx.double() - want).abs() <= _half(x.dtype) * want.abs() + room + 1e-37), "dx"
    rows = M / 64 + 4 + 96                                # a part's or group's rows in turn, up to 512 sums in 16 strips, the strips
    for got, each, extra, name in ((dw, D * h, D.abs() * d_h, "dweight"), (db, D, None, "dbias")):
        exact = each.sum(0)
        room = E * rows * each.abs().sum(0) + (0 if extra is None else extra.sum(0))
        assert torch.all((got.double() - exact).abs() <= _half(w.dtype) * exact.abs() + room + 1e-37), name


def _run(M, K, dtype, wdtype=F32, center=True, pad=0):
    print("norm", M, K, dtype, wdtype, center, flush=True)
    x, dy, w, b = _inputs(M, K, dtype, wdtype, pad)
    y, stats = reqat.layer_norm(x, w, b, center=center)
    _check_forward(x, w, b, center, y, stats)
    got = reqat.layer_norm_backward(dy, x, w, stats, center=center, bias=True)
    _check_backward(dy, x, w, stats, center, *got)
    alone = reqat.layer_norm_backward(dy, x, w, stats, center=center)
    assert alone[2] is None and torch.equal(alone[0], got[0]) and torch.equal(alone[1], got[1])
    for i in (0, 1):                                      # dx in the place of dy, and of x
        a, c = dy.clone(), x.clone()
        again = reqat.layer_norm_backward(a, c, w, stats, center=center, bias=True, out=(a, c)[i])
        assert all(torch.equal(p, q) for p, q in zip(got, again))
    z = x.clone()
    assert torch.equal(reqat.layer_norm(z, w, b, center=center, out=z)[0], y)


def _forms():
    """(type, threads, vectors a thread) of every form, with the fewest and the most vectors of a row that take it."""
    out = []
    for dtype in (BF, F32):
        for threads, most in ((64, 4), (256, 4), (512, 8)) + (((1024, 8),) if dtype == F32 else ()):
            below = {64: 0, 256: 4 * 64, 512: 4 * 256, 1024: 8 * 512}[threads]
            for vpt in range(1, most + 1):
                if vpt * threads > below:
                    out.append((dtype, threads, vpt, max(below, (vpt - 1) * threads) + 1, vpt * threads))
    return out


@pytest.mark.parametrize("rows", [5, 70, 600])
@pytest.mark.parametrize("dtype,threads,vpt,least,most", _forms())
def test_every_form(dtype, threads, vpt, least, most, rows):
    n = 8 if dtype == BF else 4
    for K in (least * n - (n - 1 if vpt > 1 or threads > 64 else 0), (most - 1) * n, most * n - 1):
        _run(rows, K, dtype, center=(rows + vpt) % 2 == 0, wdtype=BF if rows == 70 else F32, pad=0 if K == most * n else 3)


@pytest.mark.parametrize("K,dtype", [(512, BF), (2048, BF), (4096, BF), (8192, BF), (16384, BF), (32768, BF), (256, F32), (1024, F32),
                                     (4096, F32), (8192, F32), (16384, F32), (32768, F32)])
def test_full_groups(K, dtype):
    _run(67, K, dtype)


# rows beyond the workgroups of a launch, forward and backward
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,K", [(8300, 96), (8300, 1001), (2100, 4000), (2100, 3584), (1300, 8000), (1100, 13824), (1100, 16001),
                                 (1100, 20001)])
def test_more_rows_than_workgroups(M, K, dtype):
    _run(M, K, dtype)
    _run(M, K, dtype, center=False, wdtype=BF)


# parts of the columns' pass: fewer rows than parts, one more than a multiple, empty parts at the end
@pytest.mark.parametrize("M", [1, 2, 63, 64, 65, 100, 127, 129, 513, 1025])
@pytest.mark.parametrize("K,dtype", [(16387, BF), (27648, BF), (8195, F32), (20003, F32)])
def test_weight_gradients_by_columns(M, K, dtype):
    _run(M, K, dtype)
