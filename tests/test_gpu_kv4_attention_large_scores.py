"""Attention over the KV4 cache where scores are so large that the softmax is all but one-hot: finite queries give the
mean of the values whose keys score highest, at any magnitude, in one piece and in many, and the log-sum-exp where FP32
holds it.  Against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4_attention import Setup

pytestmark = pytest.mark.gpu
FLT_MAX = 3.4028234663852886e38


def one_channel(rng, nqs, heads, D, size):
    """Queries with one channel of +-size .. 2 size in every head: their scores are exact products."""
    x = np.zeros((sum(nqs), heads, D), np.float32)
    i, h = np.indices(x.shape[:2])
    x[i, h, rng.integers(0, D, x.shape[:2])] = rng.choice([-1.0, 1.0], x.shape[:2]) * np.minimum(
        size * rng.uniform(1.0, 2.0, x.shape[:2]), 3.3e38)
    return torch.from_numpy(x.reshape(sum(nqs), -1)).to(torch.bfloat16)


def check(s, got, q, nqs, scale, terms):
    """Scores are sums of `terms` products: eps bounds their error, as reqat_kv4_attention states it (FP32 sums, and 8
    roundings for the factor).  Where all other tokens lie 2 eps + 60 below the highest score, their weights (e^-60 at
    most) vanish beside the output's rounding: the mean of the highest, with the error of FP16 weights, FP32 sums and the
    bfloat16 output.  Elsewhere the output is a mean of values, so within their range.  Returns the share of such rows."""
    out, lse = (t.cpu().double().numpy() for t in got)
    D, group = s.D, q.shape[1] // (s.H * s.D)
    out = out.reshape(out.shape[0], -1, D)
    qq = q.double().numpy().reshape(out.shape)
    at, sharp, rows = 0, 0, 0
    for b, nq in enumerate(nqs):
        n = s.lens[b]
        for i in range(nq):
            m = max(0, n - nq + i + 1)
            for h in range(out.shape[1]):
                o, l = out[at + i, h], lse[at + i, h]
                where = ("sequence", b, "row", i, "head", h, "of", m)
                if m == 0:
                    assert not o.any() and l == -np.inf, where
                    continue
                k, v = s.k[b][:m, h // group], s.v[b][:m, h // group]
                z = k @ qq[at + i, h] * scale
                eps = (np.abs(k) @ np.abs(qq[at + i, h])).max() * scale * (terms + 8) * 2.0 ** -24
                top, vmax = z.max(), np.abs(v).max()
                best = z == top
                below = z[~best].max() if not best.all() else -np.inf
                steps = (64 + 4 * np.sqrt(m)) * 2.0 ** -24
                want = top + np.log(np.exp(z - top).sum())
                if abs(want) > FLT_MAX:
                    assert l == np.sign(want) * np.inf or abs(l) >= FLT_MAX * (1 - 2.0 ** -16), where + (l, want)
                else:
                    assert abs(l - want) <= eps + steps * max(1.0, abs(want)), where + (l, want, eps)
                assert np.isfinite(o).all() and np.abs(o).max() <= vmax * (1 + 2.0 ** -7), where + (o, vmax)
                rows += 1
                if top - below > 2 * eps + 60 and (terms == 1 or best.sum() == 1):
                    sharp += 1
                    mean, mass = v[best].mean(0), np.abs(v[best]).mean(0)
                    tol = 2.0 ** -8 * np.abs(mean) + mass * (2.0 ** -11 + steps) * 1.01 + m * 2.0 ** -32 * vmax
                    assert (np.abs(o - mean) <= tol).all(), where + (o, mean)
        at += nq
    return sharp / max(rows, 1)


# one piece of four waves, of eight, several pieces and their join; few queries; prompts in one piece and in several
CALLS = [([300, 33, 1, 0], [1] * 4, 2, 5), ([400], [1], 2, 5), ([5003], [1], 1, 7), ([300, 40], [5, 2], 2, 5),
         ([2500], [6], 1, 4), ([130, 40], [70, 40], 2, 3), ([1500], [65], 1, 4)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("size", [2.0 ** 22, 2.0 ** 27, 2.0 ** 29, 2.0 ** 33, 2.0 ** 50, 2.0 ** 100, 1.6e38])
def test_one_channel_queries(size, lens, nqs, H, group, D):
    print("one channel of %g: lens=%s q=%s H=%d group=%d D=%d" % (size, lens, nqs, H, group, D), flush=True)
    s = Setup(lens, H, D, 16, seed=21)
    q = one_channel(s.rng, nqs, H * group, D, size)
    assert check(s, s.run(q, nqs), q, nqs, D ** -0.5, 1) > 0.9


@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("std", [2.0 ** 12, 2.0 ** 22, 2.0 ** 28, 2.0 ** 36, 2.0 ** 110])
def test_dense_queries(std, lens, nqs, H, group):
    print("dense of %g: lens=%s q=%s H=%d group=%d" % (std, lens, nqs, H, group), flush=True)
    s = Setup(lens, H, 128, 16, seed=22)
    q = s.queries(nqs, group, std)
    assert check(s, s.run(q, nqs), q, nqs, 128 ** -0.5, 128) > 0.5


@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
def test_scores_beyond_fp32(lens, nqs, H, group):
    """Scores of either sign that FP32 does not hold, all of a row's among them."""
    print("beyond FP32: lens=%s q=%s H=%d group=%d" % (lens, nqs, H, group), flush=True)
    s = Setup(lens, H, 128, 16, seed=23, k_std=4.0)
    q = one_channel(s.rng, nqs, H * group, 128, 1.6e38)
    assert check(s, s.run(q, nqs, scale=1.0), q, nqs, 1.0, 1) > 0.9


@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
def test_rows_of_every_size_beside_each_other(lens, nqs, H, group):
    """Large rows do not touch the others of their tile, bit for bit."""
    s = Setup(lens, H, 128, 16, seed=24)
    q = s.queries(nqs, group, 2.0)
    x = q.view(len(q), -1, 128)
    large = torch.zeros(x.shape[:2], dtype=torch.bool)
    large.view(-1)[::3] = True
    mixed = torch.where(large[..., None], one_channel(s.rng, nqs, H * group, 128, 2.0 ** 40).view(x.shape), x).view(q.shape)
    print("mixed: lens=%s q=%s H=%d group=%d" % (lens, nqs, H, group), flush=True)
    want, got = s.run(q, nqs), s.run(mixed, nqs)
    assert torch.equal(got[0].view(x.shape)[~large], want[0].view(x.shape)[~large])
    assert torch.equal(got[1][~large], want[1][~large])
    assert bool(torch.isfinite(got[0]).all())
