"""Attention over the KV4 cache under tensor scales and softmax scales of any size: finite, positive FP32 numbers, where
the values and scores themselves are ordinary numbers of their formats.  Against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_cache_ref as ref
from tests.test_gpu_kv4_attention import Setup

pytestmark = pytest.mark.gpu

# one piece, the join, few queries, a prompt in one piece and in several
CALLS = [([300, 33, 1, 0], [1] * 4, 2, 5), ([2049], [1], 1, 7), ([300, 40], [5, 2], 2, 5), ([130, 40], [70, 40], 2, 3),
         ([1200], [65], 1, 4)]


def run(gk, gv, lens, nqs, H, group, D, scale=None, seed=31, least=0x20, most=0x47):
    """Random codes, scale bytes least .. most (0x20 .. 0x47: 2^-3 to 3.75), queries for scores of a standard deviation of 2."""
    scale = D ** -0.5 if scale is None else scale
    gk, gv, scale = (float(np.float32(x)) for x in (gk, gv, scale))
    print("gk=%g gv=%g scale=%g lens=%s q=%s D=%d" % (gk, gv, scale, lens, nqs, D), flush=True)
    s = Setup(lens, H, D, 16, seed=seed, gk=gk, gv=gv)
    for i, (g, values) in enumerate(((gk, s.k), (gv, s.v))):
        for b, n in enumerate(lens):
            c = s.rng.integers(0, 16, (n, H, D)).astype(np.uint8)
            t = s.rng.integers(least, most + 1, (n, H, D // 16)).astype(np.uint8)
            if n:
                j = np.arange(n)
                at = (s.table[b, j // s.P], j % s.P)
                s.arrays[2 * i][at], s.arrays[2 * i + 1][at] = c, t
            values[b] = ref.values(c, t, g)
    s.upload()
    rms = math.sqrt(np.mean(np.concatenate([k.ravel() for k in s.k]) ** 2)) if gk > 1e-30 else \
        gk * math.sqrt(np.mean((np.concatenate([k.ravel() for k in s.k]) / gk) ** 2))
    q = s.queries(nqs, group, 1.0).double() * (2.0 / (rms * math.sqrt(D)) / scale)
    q = q.to(torch.bfloat16)
    assert bool(torch.isfinite(q).all()) and bool(q.any())
    out, lse = (t.cpu().double().numpy() for t in s.run(q, nqs, scale=scale))
    out = out.reshape(out.shape[0], -1, D)
    qq = q.double().numpy().reshape(out.shape)
    up = 2.0 ** -math.frexp(gv)[1]                  # the bounds are those of values near one
    at = 0
    for b, nq in enumerate(nqs):
        v = s.v[b] * up
        o, l, mass, reach = ref.attention(qq[at:at + nq], s.k[b], v, True, scale)
        tol, ltol = ref.bounds(o, l, mass, reach, max(1, lens[b]), D, np.abs(v).max() if lens[b] else 0.0)
        tol = tol + 2.0 ** -134 * 1.01 * up         # half a step of the smallest bfloat16 numbers
        for name, g, w, t in (("out", out[at:at + nq] * up, o, tol), ("lse", lse[at:at + nq], l, ltol)):
            with np.errstate(invalid="ignore"):
                bad = np.argwhere(~((np.abs(g - w) <= t) | (g == w)))
            assert bad.size == 0, (name, b, len(bad), bad[:3], g[tuple(bad[0])], w[tuple(bad[0])], t[tuple(bad[0])])
        at += nq


@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("gv", [2.0 ** 116, 1.9 * 2.0 ** 123, 2.0 ** -110, 2.0 ** -126, 3.0e-39])
def test_scale_of_the_values(gv, lens, nqs, H, group):
    run(2.0 ** -6, gv, lens, nqs, H, group, 128)


@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("gk,scale", [(2.0 ** 100, None), (1.7 * 2.0 ** 118, None), (2.0 ** -100, None),
                                      (2.0 ** -120, None), (2.0 ** -127, 64.0)])
def test_scale_of_the_keys(gk, scale, lens, nqs, H, group):
    run(gk, 0.37, lens, nqs, H, group, 128, scale)


@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("gk,scale", [(2.0 ** -6, 1e30), (2.0 ** -6, 1e-30), (2.0 ** -20, 3e38), (2.0 ** 60, 1e-42),
                                      (2.0 ** -60, 1e38)])
def test_scale_of_the_softmax(gk, scale, lens, nqs, H, group):
    run(gk, 1.0, lens, nqs, H, group, 128, scale)


def test_narrow_heads():
    for gk, gv in ((2.0 ** 118, 2.0 ** -126), (2.0 ** -120, 2.0 ** 120)):
        run(gk, gv, [2049, 7], [1, 1], 2, 4, 64)
        run(gk, gv, [700], [65], 1, 4, 64)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("least,most", [(1, 7), (1, 20), (0x70, 0x7E)])
def test_block_scales_at_the_ends(least, most, lens, nqs, H, group, D):
    """E4M3 subnormals (2^-9 to 7 2^-9) and the numbers next to them, and the largest."""
    run(2.0 ** -3, 2.0 ** -4, lens, nqs, H, group, D, seed=32, least=least, most=most)
