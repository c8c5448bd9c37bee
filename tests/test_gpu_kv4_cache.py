"""Writing the paged KV4 cache and reading it back, byte for byte against the
plain definitions: head sizes and counts, page sizes, rotation and shift, scales
that are and are not powers of two, padding, strided rows, midpoints and
non-finite values, pages beyond 2^32 bytes; every byte outside the named slots
stays as it was."""
import numpy as np
import pytest
import torch

from paper_2606_15682_amd import reqat
from paper_2606_15682_amd import workloads as wl
from tests import kv4_cache_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rope_tables(P, D, seed=5):
    a = np.random.default_rng(seed).uniform(-np.pi, np.pi, (P, D // 2))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def make_cache(pages, P, H, D, gk=2.0 ** -6, gv=2.0 ** -6, shift=None, fill=0xA5):
    c = reqat.Kv4Cache(pages, P, H, D, k_scale=gk, v_scale=gv, device=DEV,
                       k_shift=None if shift is None else torch.from_numpy(shift).to(DEV))
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        t.fill_(fill)
    return c


def read(c):
    return ref.unpack(*(t.cpu().numpy() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales)),
                      c.num_pages, c.page_size, c.kv_heads, c.head_dim)


def bf16(rng, shape, std=1.0):
    """bfloat16 values as (device tensor, FP32 array)"""
    b = wl.bf16_bits(torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16))
    return b, ref.bf16_f32(b)


def dev(bits, pad=0):
    """The bfloat16 tensor of bit patterns, as columns of wider rows when pad > 0."""
    t = wl.from_bits(bits)
    if pad:
        wide = torch.full((t.shape[0], t.shape[1] + 2 * pad), float("nan"), dtype=torch.bfloat16)
        wide[:, pad:pad + t.shape[1]] = t
        return wide.to(DEV)[:, pad:pad + t.shape[1]]
    return t.to(DEV)


def check_append(T, H, Hq, D, P, gk=2.0 ** -6, gv=2.0 ** -6, rope=True, shifted=True, pad=0, kbits=None, vbits=None,
                 positions=None, seed=0, inplace=False):
    print("append T=%d H=%d Hq=%d D=%d P=%d gk=%r gv=%r rope=%s shift=%s pad=%d" % (T, H, Hq, D, P, gk, gv, rope, shifted,
                                                                                  pad), flush=True)
    rng = np.random.default_rng(seed + 7 * T + D)
    pages = -(-(T + 5) // P) + 2
    kb, k = bf16(rng, (T, H * D)) if kbits is None else (kbits, ref.bf16_f32(kbits))
    vb, v = bf16(rng, (T, H * D)) if vbits is None else (vbits, ref.bf16_f32(vbits))
    qb, q = bf16(rng, (T, max(Hq, 1) * D), 3.0)
    shift = (rng.standard_normal(H * D) * 2).astype(np.float32) if shifted else None
    slots = rng.permutation(pages * P)[:T].astype(np.int64)
    if T > 2:
        slots[T // 2] = -1
        slots[T // 3] = pages * P
    cos, sin = rope_tables(97, D)
    pos = rng.integers(0, 97, T).astype(np.int32) if positions is None else positions
    c = make_cache(pages, P, H, D, gk, gv, shift)
    before = read(c)
    kw = {}
    if rope:
        kw = dict(rope=(torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)),
                  positions=torch.from_numpy(pos).to(DEV))
        if Hq:
            kw["q"] = dev(qb, pad)
            if inplace:
                kw["q_out"] = kw["q"]
    got_q = reqat.kv4_append(c, dev(kb, pad), dev(vb, pad), torch.from_numpy(slots).to(DEV), **kw)
    torch.cuda.synchronize()
    assert (got_q is None) == (not (rope and Hq))
    with np.errstate(all="ignore"):
        kk, qq = k.reshape(T, H, D), q.reshape(T, -1, D)
        if rope:
            ok = (pos >= 0) & (pos < 97)
            cs, sn = (np.where(ok[:, None], t[np.clip(pos, 0, 96)], np.float32("nan")) for t in (cos, sin))
            kk, qq = ref.rotate(kk, cs, sn), ref.rotate(qq, cs, sn)
        if shifted:
            kk = kk - shift.reshape(H, D)
        want = [x.copy() for x in before]
        kc, ks = ref.quantize(kk, gk)
        vc, vs = ref.quantize(v.reshape(T, H, D), gv)
    keep = (slots >= 0) & (slots < pages * P)
    at = (slots[keep] // P, slots[keep] % P)
    for w, new in zip(want, (kc, ks, vc, vs)):
        w[at] = new[keep]
    for name, g, w in zip(("k codes", "k scales", "v codes", "v scales"), read(c), want):
        bad = np.argwhere(g != w)
        assert bad.size == 0, (name, len(bad), bad[:3], g[tuple(bad[0])], w[tuple(bad[0])])
    if rope and Hq:
        g = ref.bf16_f32(wl.bf16_bits(got_q.cpu())).astype(np.float64)
        assert np.array_equal(g, ref.to_bf16(qq).reshape(T, -1), equal_nan=True)
    return c, slots


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,H,Hq,P", [(1, 1, 1, 16), (2, 2, 12, 16), (5, 3, 6, 64), (300, 8, 40, 32), (777, 1, 7, 128),
                                      (33, 4, 28, 1024)])
def test_append_rotated(T, H, Hq, P, D):
    check_append(T, H, Hq, D, P, pad=0 if T % 2 else 24)


@pytest.mark.parametrize("rope,shifted", [(False, False), (False, True), (True, False)])
@pytest.mark.parametrize("gk,gv", [(2.0 ** -6, 2.0 ** -9), (0.0123, 1.0 / 3.0), (2.0 ** -126, 3.0e-39), (2.0 ** 101, 1e30)])
def test_append_scales(rope, shifted, gk, gv):
    check_append(129, 2, 4, 128, 16, gk, gv, rope, shifted, pad=8)


def test_append_without_queries_and_in_place():
    check_append(40, 2, 0, 128, 32)
    check_append(40, 2, 6, 64, 32, inplace=True, pad=8)


def test_append_positions_outside_the_tables():
    pos = np.arange(50, dtype=np.int32) % 97
    pos[[0, 7, 49]] = [-1, 97, 2 ** 31 - 1]
    check_append(50, 2, 4, 128, 16, positions=pos)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g", [2.0 ** -6, 0.0317])
def test_append_special_values(D, g):
    """Midpoints and their neighbours, zeros of both signs, subnormals, infinities and NaN."""
    rng = np.random.default_rng(3)
    T, H = 96, 2
    s = ref.E4M3[rng.integers(1, 127, (T, H * D // 16, 1))]
    m = rng.choice([0.25, 0.75, 1.25, 1.75, 2.25, 2.75, 3.25, 0.0, 3.5, 1.0], (T, H * D // 16, 16))
    m[..., 0] = 3.5
    x = (m * s * g * rng.choice([-1.0, 1.0], m.shape)).astype(np.float32).reshape(T, H * D)
    bits = wl.bf16_bits(torch.from_numpy(x).to(torch.bfloat16)).copy()
    near = rng.integers(-1, 2, bits.shape).astype(np.int32)
    bits = np.where((bits & 0x7FFF) > 2, bits + near, bits).astype(np.uint16)
    bits[3, :40] = 0
    bits[4, :40] = 0x8000
    bits[5, 3], bits[6, 20], bits[7, 33] = 0x7F80, 0xFF80, 0x7FC1
    bits[8, :16] = np.arange(16)
    bits[9] = 0x7F7F
    check_append(T, H, 2, D, 16, g, g, rope=False, shifted=False, kbits=bits, vbits=bits[::-1].copy())
    check_append(T, H, 2, D, 16, g, g, rope=True, shifted=True, kbits=bits, vbits=bits[::-1].copy())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gk,gv", [(2.0 ** -6, 2.0 ** -6), (0.0123, 1.0 / 3.0), (2.0 ** -127, 2.0 ** 120)])
@pytest.mark.parametrize("shifted", [False, True])
def test_gather_every_code_and_scale(D, gk, gv, shifted):
    """All 256 scale bytes of both signs of NaN with all codes, any slots, padding, strided outputs."""
    print("gather D=%d gk=%r gv=%r shift=%s" % (D, gk, gv, shifted), flush=True)
    rng = np.random.default_rng(11)
    H, P, pages = 3, 32, 9
    sh = (rng.standard_normal(H * D) * 2).astype(np.float32) if shifted else None
    c = make_cache(pages, P, H, D, gk, gv, sh)
    arrays = [rng.integers(0, 16, (pages, P, H, D)).astype(np.uint8), rng.integers(0, 128, (pages, P, H, D // 16)).astype(np.uint8),
              rng.integers(0, 16, (pages, P, H, D)).astype(np.uint8), rng.integers(0, 128, (pages, P, H, D // 16)).astype(np.uint8)]
    for t, b in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales), ref.pack(*arrays)):
        t.copy_(torch.from_numpy(b))
    slots = np.concatenate([rng.permutation(pages * P), [-1, 3, 3, pages * P, 2 ** 62, -2 ** 62]]).astype(np.int64)
    T = len(slots)
    ko, vo = (torch.full((T, H * D + 16), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    out = (ko[:, 8:8 + H * D], vo[:, 8:8 + H * D])
    reqat.kv4_gather(c, torch.from_numpy(slots).to(DEV), add_shift=True, out=out)
    plain = reqat.kv4_gather(c, torch.from_numpy(slots).to(DEV))
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < pages * P)
    at = np.clip(slots, 0, pages * P - 1)
    k = ref.values(arrays[0], arrays[1], gk).reshape(pages * P, H * D)[at]
    v = ref.values(arrays[2], arrays[3], gv).reshape(pages * P, H * D)[at]
    ks = (k.astype(np.float32) + sh) if shifted else k
    for name, got, want in (("k", plain[0], k), ("v", plain[1], v), ("k + m", out[0], ks), ("v", out[1], v)):
        g = ref.bf16_f32(wl.bf16_bits(got.cpu())).astype(np.float64)
        w = np.where(ok[:, None], ref.to_bf16(want), 0.0)
        bad = np.argwhere(~((g == w) | (np.isnan(g) & np.isnan(w))))
        assert bad.size == 0, (name, len(bad), bad[:3], g[tuple(bad[0])], w[tuple(bad[0])])
    for o in (ko, vo):
        assert bool((o[:, :8] == 7.0).all()) and bool((o[:, 8 + H * D:] == 7.0).all())


def test_append_then_gather_matches_the_fakequant():
    """Without rotation the cache holds what reqat_fakequant_kv4 of the same rows gives."""
    rng = np.random.default_rng(2)
    T, H, D = 500, 4, 128
    kb, _ = bf16(rng, (T, H * D))
    vb, _ = bf16(rng, (T, H * D))
    sh = (rng.standard_normal(H * D)).astype(np.float32)
    c = make_cache(40, 16, H, D, 0.02, 2.0 ** -7, sh)
    slots = torch.randperm(640, device=DEV)[:T]
    reqat.kv4_append(c, dev(kb), dev(vb), slots)
    k, v = reqat.kv4_gather(c, slots)
    assert torch.equal(k, reqat.fakequant_kv4(dev(kb), c.k_shift, tensor_scale=c.k_scale)[0])
    assert torch.equal(v, reqat.fakequant_kv4(dev(vb), None, tensor_scale=c.v_scale)[0])


def test_no_tokens():
    c = make_cache(1, 16, 2, 128)
    e = torch.empty((0, 256), dtype=torch.bfloat16, device=DEV)
    s = torch.empty(0, dtype=torch.int64, device=DEV)
    assert reqat.kv4_append(c, e, e, s) is None
    assert reqat.kv4_gather(c, s)[0].shape == (0, 256)


def test_pages_beyond_32_bits():
    """Codes of more than 2^32 bytes: the last pages, and the same ones modulo 2^32, stay apart."""
    H, D, P = 8, 128, 1024
    pages = (1 << 32) // (H * P * D // 2) + 3
    print("cache of %d pages, %.1f GB" % (pages, 2 * pages * H * P * (D // 2 + D // 16) / 1e9), flush=True)
    c = reqat.Kv4Cache(pages, P, H, D, k_scale=2.0 ** -6, v_scale=2.0 ** -6, device=DEV)
    rng = np.random.default_rng(9)
    kb, _ = bf16(rng, (64, H * D))
    vb, _ = bf16(rng, (64, H * D))
    last = torch.arange(pages * P - 64, pages * P, device=DEV)
    reqat.kv4_append(c, dev(kb), dev(vb), last)
    k, v = reqat.kv4_gather(c, last)
    assert torch.equal(k, reqat.fakequant_kv4(dev(kb), None, tensor_scale=c.k_scale)[0])
    assert torch.equal(v, reqat.fakequant_kv4(dev(vb), None, tensor_scale=c.v_scale)[0])
    assert int(torch.count_nonzero(c.k_codes)) == int(torch.count_nonzero(c.k_codes[-H * P * D // 2:]))
    low = torch.arange(64, device=DEV)
    assert not bool(reqat.kv4_gather(c, low)[0].any())
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV)
    # the last page's first tokens hold zeros, its last 64 the keys: a query over all of them
    q = dev(bf16(rng, (1, H * D))[0])
    out = reqat.kv4_attention(q, c, table, torch.tensor([P], dtype=torch.int32, device=DEV))
    kk = torch.cat([torch.zeros((P - 64, H * D), device=DEV), k.float()]).double().cpu().numpy().reshape(P, H, D)
    vv = torch.cat([torch.zeros((P - 64, H * D), device=DEV), v.float()]).double().cpu().numpy().reshape(P, H, D)
    qq = q.double().cpu().numpy().reshape(1, H, D)
    want = ref.attention(qq, kk, vv, True, D ** -0.5)
    tol, _ = ref.bounds(*want, P, D, np.abs(vv).max())
    assert bool((np.abs(out.double().cpu().numpy().reshape(1, H, D) - want[0]) <= tol).all())
