"""The paged KV4 cache in plain numpy and 64 bits, from the definitions in
include/reqat.h: quantization of FP32 rows, the byte layout of pages, rotation,
attention.  Shares no code with the library or the oracle."""
import numpy as np

E4M3 = np.array([(m / 8.0 + (1.0 if e else 0.0)) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)])
E4M3[127] = np.nan


def bf16_f32(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)


def to_bf16(x):
    """Nearest bfloat16 of FP64 or FP32 values (ties to even, one rounding), as FP64."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        _, e = np.frexp(x)
        unit = np.ldexp(1.0, np.maximum(e - 8, -133))
        r = np.round(x / unit) * unit
        r = np.where(np.abs(r) >= 2.0 ** 128, np.sign(r) * np.inf, r)
    return np.where(np.isfinite(x), r, x)


def quantize(d, g):
    """Codes (uint8 0..15) and E4M3 bytes of the blocks of 16 along the last axis of d (FP32); all bounds and
    thresholds are exact in FP64."""
    g = float(np.float32(g))
    d = np.asarray(d, np.float32).astype(np.float64)
    blk = d.reshape(d.shape[:-1] + (d.shape[-1] // 16, 16))
    a = np.abs(blk)
    bad = ~np.isfinite(blk).all(-1)
    amax = np.where(bad, 0.0, np.where(np.isfinite(a), a, 0.0).max(-1))
    byte = np.searchsorted(3.5 * E4M3[1:127] * g, amax, side="left") + 1
    byte = np.where(amax == 0.0, 0, np.minimum(byte, 126))
    s = (E4M3[byte] * g)[..., None]
    code = np.zeros(blk.shape, np.uint8)
    for i in range(7):
        t = (0.5 * i + 0.25) * s
        code += ((a > t) if i % 2 == 0 else (a >= t)).astype(np.uint8)
    code = np.where((byte == 0)[..., None], 0, code) + 8 * np.signbit(blk)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(d.shape).astype(np.uint8), np.where(bad, 127, byte).astype(np.uint8)


def values(codes, sbytes, g):
    c = codes.astype(np.int64)
    v = np.where(c & 8, -0.5, 0.5) * (c & 7)
    v = v.reshape(v.shape[:-1] + (v.shape[-1] // 16, 16)) * (E4M3[sbytes & 127] * float(np.float32(g)))[..., None]
    return v.reshape(codes.shape)


def unpack(kc, ks, vc, vs, pages, P, H, D):
    """Bytes of the four arrays -> (k codes, k scales, v codes, v scales) as [pages, P, H, D or D / 16]."""
    def nibbles(b):
        return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (-1,))
    k = nibbles(kc.reshape(pages, H, P, D // 2)).transpose(0, 2, 1, 3)
    s = ks.reshape(pages, H, P, D // 16).transpose(0, 2, 1, 3)
    v = nibbles(vc.reshape(pages, H, P // 4, D // 8, 4, 4)).transpose(0, 2, 4, 1, 3, 5).reshape(pages, P, H, D)
    t = vs.reshape(pages, H, P // 4, D // 16, 4).transpose(0, 2, 4, 1, 3).reshape(pages, P, H, D // 16)
    return k, s, v, t


def pack(k, s, v, t):
    """The inverse of unpack."""
    pages, P, H, D = k.shape
    def halves(c):
        return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
    kc = halves(k.transpose(0, 2, 1, 3))
    vc = halves(v).reshape(pages, P // 4, 4, H, D // 8, 4).transpose(0, 3, 1, 4, 2, 5)
    vs = t.reshape(pages, P // 4, 4, H, D // 16).transpose(0, 3, 1, 4, 2)
    return tuple(np.ascontiguousarray(x).reshape(-1) for x in (kc, s.transpose(0, 2, 1, 3), vc, vs))


def rotate(x, cos, sin):
    """x [T, heads, D] FP32, cos and sin [T, D / 2] FP32; every operation rounded to FP32."""
    h = x.shape[-1] // 2
    lo, hi = x[..., :h].astype(np.float32), x[..., h:].astype(np.float32)
    c, s = cos[:, None, :], sin[:, None, :]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def attention(q, k, v, causal, scale):
    """q [nq, Hq, D], k and v [n, H, D], FP64 -> out [nq, Hq, D], lse [nq, Hq], and for the error bound
    sum p |v| / sum p [nq, Hq, D] and max_j scale sum_d |q_d k_jd| [nq, Hq].  Hidden tokens are left out."""
    nq, Hq, D = q.shape
    n, H, _ = k.shape
    out, lse = np.zeros((nq, Hq, D)), np.full((nq, Hq), -np.inf)
    mass, reach = np.zeros((nq, Hq, D)), np.zeros((nq, Hq))
    with np.errstate(all="ignore"):
        for h in range(Hq):
            kh, vh = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
            for i in range(nq):
                m = max(0, n - nq + i + 1) if causal else n
                if m == 0:
                    continue
                z = kh[:m] @ q[i, h] * scale
                top = z.max()
                p = np.exp(z - top)
                tot = p.sum()
                out[i, h] = p @ vh[:m] / tot
                lse[i, h] = top + np.log(tot)
                mass[i, h] = p @ np.abs(vh[:m]) / tot
                reach[i, h] = (np.abs(kh[:m]) @ np.abs(q[i, h])).max() * scale
    return out, lse, mass, reach


def bounds(out, lse, mass, reach, n, D, vmax):
    """Allowed errors of out and lse, from the roundings that reqat_kv4_attention states: FP32 scores (D + 8 roundings
    of at most 2^-24 of the sum of magnitudes, each moving p by as much), the FP16 weights (2^-11; 2^-32 of the largest
    below their normal range, and n of them), FP32 sums (errors of either sign: 4 sqrt(n) roundings, and 64 for the
    exponentials and the rescaling), and the bfloat16 output."""
    eps = reach * (D + 8) * 2.0 ** -24
    rel = 2.0 ** -11 + 2.0 * eps[..., None] + (64 + 4 * np.sqrt(n)) * 2.0 ** -24
    return 2.0 ** -8 * np.abs(out) + mass * rel * 1.01 + n * 2.0 ** -32 * vmax + 1e-30, \
        eps + (64 + 4 * np.sqrt(n)) * 2.0 ** -24 * np.maximum(1.0, np.abs(lse))
