"""GPU: infinities and NaN in rows of the norms, at every kind of place: what they give is the formula's, whatever the channel and
the row's length."""
import math

import pytest
import torch

from paper_2606_15682_amd import reqat

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32

# lengths with and without threads that have no elements in their last vector, and odd ones
LENGTHS = [3, 7, 8, 9, 100, 511, 513, 1024, 1536, 1540, 2049, 3584, 5120, 5121, 6145, 8193, 9000, 13824, 16385, 20001]


def _expected(x, w, center, eps=1e-6):
    z = x.double()
    mu = z.mean(1, keepdim=True) if center else torch.zeros((), dtype=torch.float64)
    d = z - mu
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    return d * rstd * w.double(), rstd[:, 0]


@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", LENGTHS)
def test_forward(K, dtype, center):
    print("norm with infinities", K, dtype, center, flush=True)
    places = sorted({0, 1, 2, 7, K // 2, K - 2, K - 1} & set(range(K)))
    g = torch.Generator().manual_seed(K)
    x = torch.randn((2 * len(places) + 1, K), generator=g).to(dtype)
    for i, j in enumerate(places):
        x[2 * i, j] = math.inf if i % 2 else -math.inf
        x[2 * i + 1, j] = math.nan
    w = 1.0 + 0.1 * torch.randn(K, generator=g)
    want, rstd = _expected(x, w, center)
    y, stats = reqat.layer_norm(x.to(DEV), w.to(DEV), center=center)
    y, stats = y.double().cpu(), stats.double().cpu()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(torch.isnan(stats[:, 1]), torch.isnan(rstd))
    assert torch.equal(stats[:, 1] == 0, rstd == 0)
    infinite = rstd == 0                                   # without centring: zeros but at the infinity, 0 times Inf
    assert bool(infinite.any()) == (not center)
    assert torch.equal(y[infinite].nan_to_num(1.0), want[infinite].nan_to_num(1.0))


@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", LENGTHS)
def test_backward(K, dtype, center):
    """An infinite or NaN gradient makes its row's dx NaN and its own column of dweight, no other row and no other column."""
    g = torch.Generator().manual_seed(K)
    x, dy = (torch.randn((5, K), generator=g).to(dtype).to(DEV) for _ in range(2))
    w = (1.0 + 0.1 * torch.randn(K, generator=g)).to(DEV)
    stats = reqat.layer_norm(x, w, center=center)[1]
    dx, dw, db = reqat.layer_norm_backward(dy, x, w, stats, center=center, bias=True)
    for j, bad in ((0, math.inf), (K - 1, math.nan), (K // 2, -math.inf)):
        other = dy.clone()
        other[3, j] = bad
        dx2, dw2, db2 = reqat.layer_norm_backward(other, x, w, stats, center=center, bias=True)
        rows = torch.tensor([0, 1, 2, 4], device=DEV)
        assert torch.equal(dx2[rows], dx[rows]) and torch.isnan(dx2[3, j])
        columns = torch.arange(K, device=DEV) != j
        assert torch.equal(dw2[columns], dw[columns]) and torch.equal(db2[columns], db[columns])
        assert not torch.isfinite(dw2[j]) and not torch.isfinite(db2[j])
