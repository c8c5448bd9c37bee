// Quantization of one 16-channel block of the KV4 format: the E4M3 scale byte and the
// E1M2 codes of 16 shifted values under a global scale.  For the tensor quantizer
// (kv4.hip) and the paged cache's writer (kv4_cache.hip).
#pragma once

#include "fp4_device.h"

namespace reqat {

// Smallest positive finite E4M3 s with amax <= 3.5 * s * g (0x7E when none).
__device__ __forceinline__ uint32_t kv4_scale_byte(double a, double g) {
    uint32_t b = e4m3_ceil_byte(a / (3.5 * g));
    if (b < 0x7Eu && !(a <= 3.5 * (double)e4m3_value(b) * g)) b += 1u;
    else if (b > 1u && a <= 3.5 * (double)e4m3_value(b - 1u) * g) b -= 1u;
    return b;
}

// FP32 counterpart for a power-of-two g = 2^kg in [2^-126, 2^100]: q = a / (3.5 g)
// to within a few ulp, its E4M3 ceiling, then one exact correction.  Every
// bound 3.5 * s * g has at most 7 significant bits and lies in
// [7 * 2^-136, 1568 * 2^100], so it is exact in FP32 (subnormals included).
__device__ __forceinline__ uint32_t kv4_scale_byte_f32(float a, float g, int kg) {
    const float q = __builtin_ldexpf(a * (2.0f / 7.0f), -kg);
    uint32_t b;
    if (!(q <= 448.0f)) {
        b = 0x7Eu;
    } else if (q <= 0x1p-9f) {
        b = 0x01u;
    } else {
        const uint32_t qb = bits_from_f32(q);           // normal: q > 2^-9
        int E = (int)(qb >> 23) - 127;
        if (E < -6) {
            b = (uint32_t)__builtin_ceilf(q * 0x1p9f);  // E4M3 subnormals: multiples of 2^-9 (1..8)
        } else {
            uint32_t m = ((qb & 0x7FFFFFu) + 0xFFFFFu) >> 20;   // ceil of the top three mantissa bits
            if (m == 8u) {
                m = 0u;
                E += 1;
            }
            b = ((uint32_t)(E + 7) << 3) | m;
            b = b > 0x7Eu ? 0x7Eu : b;
        }
    }
    if (b < 0x7Eu && !(a <= 3.5f * e4m3_value(b) * g)) b += 1u;
    else if (b > 1u && a <= 3.5f * e4m3_value(b - 1u) * g) b -= 1u;
    return b;
}

// E1M2 magnitude code (0..7) of |v| / S, nearest with ties to the even code.
__device__ __forceinline__ uint32_t e1m2_mag(double a, double S) {
    uint32_t m = 7u;
#pragma unroll
    for (int i = 6; i >= 0; --i) {
        const double t = (0.5 * i + 0.25) * S;
        if (a < t || (a == t && (i & 1) == 0)) m = (uint32_t)i;
    }
    return m;
}

// The same with FP32 thresholds, exact when S = s * g is a power-of-two
// multiple of an E4M3 value inside the FP32 range: (0.5 i + 0.25) * S has at
// most 8 significant bits and lies in [2^-137, 2^111].
__device__ __forceinline__ uint32_t e1m2_mag_f32(float a, float S) {
    uint32_t m = 7u;
#pragma unroll
    for (int i = 6; i >= 0; --i) {
        const float t = (0.5f * (float)i + 0.25f) * S;
        if (a < t || (a == t && (i & 1) == 0)) m = (uint32_t)i;
    }
    return m;
}

// The global scale g as the element paths use it: the FP32 path needs a
// power of two in [2^-126, 2^100] (every computed g is a power of two), so
// that every threshold and decoded value is exact in FP32.
struct Kv4G {
    float g;
    double gd;
    bool f32;
    int kg;
};

__device__ __forceinline__ Kv4G kv4_make_g(float g) {
    Kv4G G;
    G.g = g;
    G.gd = (double)g;
    const uint32_t gb = bits_from_f32(g);
    G.f32 = (gb & 0x807FFFFFu) == 0u && gb >= 0x00800000u && gb <= ((100u + 127u) << 23);
    G.kg = (int)(gb >> 23) - 127;
    return G;
}

// Exact element codes of one block (sign in bit 3, magnitude 0..7) by
// threshold comparisons: FP32 thresholds for a power-of-two g, FP64 otherwise.
__device__ __forceinline__ void kv4_exact_codes(const float (&d)[16], bool bad, uint32_t sbyte, const Kv4G &G,
                                                double S, float Sf, uint32_t (&c)[16]) {
    if (G.f32) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t sign = (bits_from_f32(d[j]) >> 28) & 8u;
            c[j] = bad ? 0u : (sbyte == 0u ? sign : (e1m2_mag_f32(__builtin_fabsf(d[j]), Sf) | sign));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t sign = (bits_from_f32(d[j]) >> 28) & 8u;
            c[j] = bad ? 0u : (sbyte == 0u ? sign : (e1m2_mag(__builtin_fabs((double)d[j]), S) | sign));
        }
    }
}

// Packs eight codes (sign in bit 3, magnitude 0..7 = |c|) of the integral
// values c[0..8) into a word, code j in bits 4j..4j+3: magnitudes converted
// into bytes (even j in one word, odd j in another), signs gathered from the
// top bytes of the FP32 patterns.
__device__ __forceinline__ uint32_t kv4_pack8(const float *c) {
    uint32_t pe = 0u, po = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        pe = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_fabsf(c[2 * k]), k, pe);
        po = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_fabsf(c[2 * k + 1]), k, po);
    }
    // top byte of c[2k] (resp. c[2k+1]) into byte k; 0x0C selects a zero byte
    const uint32_t se = __builtin_amdgcn_perm(bits_from_f32(c[2]), bits_from_f32(c[0]), 0x0C0C0703u) |
                        __builtin_amdgcn_perm(bits_from_f32(c[6]), bits_from_f32(c[4]), 0x07030C0Cu);
    const uint32_t so = __builtin_amdgcn_perm(bits_from_f32(c[3]), bits_from_f32(c[1]), 0x0C0C0703u) |
                        __builtin_amdgcn_perm(bits_from_f32(c[7]), bits_from_f32(c[5]), 0x07030C0Cu);
    return (pe | (po << 4)) | ((se >> 4) & 0x08080808u) | (so & 0x80808080u);
}

// Largest |d| of a block as an FP32 pattern.  The IEEE maximum propagates NaN,
// so a block with a NaN or an infinity gives a pattern >= 0x7F800000.
__device__ __forceinline__ uint32_t kv4_block_max(const float (&d)[16]) {
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < 16; ++j) m = __builtin_elementwise_maximum(m, __builtin_fabsf(d[j]));
    return bits_from_f32(m);
}

// A rounded block: its scale byte, S = s g and H = S / 2 in FP32, and the code of d[j]
// as the integral value cf[j], unless `exact` says that the thresholds have to decide.
struct Kv4Rounded {
    uint32_t sbyte;
    bool bad, exact;
    float Sf, H, cf[16];
};

// Rounds a block (its 16 shifted values d, am = the largest |d| pattern, NaN and
// Inf included) under G.
//
// Fast path (power-of-two g, finite block, H = s g / 2 zero or a normal FP32
// value, am <= 7 H, i.e. the scale did not saturate): the code magnitude is
// the integer nearest |d| / H, ties to even (at most 7).  q = d * rcp(H) is
// within 2^-19 of d / H (the reciprocal's ulp and one rounding, |q| <= 7), so
// rint(q) is the code with d's sign (-0 for a small negative d) unless d / H
// lies within 2^-19 of a half-integer; q - rint(q) is exact, and a block with
// some |q - rint(q)| >= 0.5 - 2^-17 takes the threshold path instead.  The
// fake-quant value c * H has at most 7 significant bits and is normal or
// zero, so its top 16 bits are the bfloat16 value.
//
// kBf16 (no shift: d is a bfloat16 value, 8 significant bits): exact midpoints
// are common, about one element in 60 of normal data, and nearly every wave took the
// threshold path for some lane.  Here a quotient that is not a half-integer
// lies at least 2^-10 from every one: in |d - mid H| the two are multiples of 2^a
// (d = D 2^a, 128 <= D < 256 or d subnormal) and 2^(e-1) (H = h 2^e, h <= 15), so
// a difference is at least H / 30 or, near the midpoint, about H / 512.  So q is
// rounded to a multiple of 2^-12 (by adding 3072: the sum lies in [2048, 4096)),
// which gives a half-integer exactly where d / H is one and keeps the side
// elsewhere; then rint decides as above, ties included, and no block is left
// undecided.  The pass over values of a 32768 x 1024 cache slice: 40 -> 26 us.
template <bool kBf16>
__device__ __forceinline__ Kv4Rounded kv4_round(const float (&d)[16], uint32_t am, const Kv4G &G) {
    Kv4Rounded R;
    const bool bad = am >= 0x7F800000u;
    const uint32_t sbyte = bad ? 0x7Fu
                           : am == 0u ? 0u
                           : G.f32 ? kv4_scale_byte_f32(f32_from_bits(am), G.g, G.kg)
                                   : kv4_scale_byte((double)f32_from_bits(am), G.gd);
    const float Sf = e4m3_value(sbyte) * G.g;               // exact on the FP32 path
    const float H = 0.5f * Sf;
    const bool fast_ok = G.f32 && !bad && (sbyte == 0u || (H >= 0x1p-126f && f32_from_bits(am) <= 7.0f * H));
    const float rh = (fast_ok && sbyte != 0u) ? __builtin_amdgcn_rcpf(H) : 0.0f;
    float emax = 0.0f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        if constexpr (kBf16) {
            const float q = __builtin_fmaf(d[j], rh, 3072.0f) - 3072.0f;
            R.cf[j] = __builtin_copysignf(__builtin_rintf(q), d[j]);
        } else {
            const float q = d[j] * rh;
            R.cf[j] = __builtin_rintf(q);
            emax = __builtin_fmaxf(emax, __builtin_fabsf(q - R.cf[j]));
        }
    }
    R.exact = !fast_ok || emax >= 0.5f - 0x1p-17f;
    R.sbyte = sbyte;
    R.bad = bad;
    R.Sf = Sf;
    R.H = H;
    return R;
}

// The block's codes as two words, code j of each in bits 4j..4j+3.
__device__ __forceinline__ uint2 kv4_codes(const float (&d)[16], const Kv4Rounded &R, const Kv4G &G) {
    uint32_t lo = kv4_pack8(R.cf), hi = kv4_pack8(R.cf + 8);
    if (R.exact) {
        uint32_t c[16];
        kv4_exact_codes(d, R.bad, R.sbyte, G, (double)e4m3_value(R.sbyte) * G.gd, R.Sf, c);
        lo = 0;
        hi = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo |= c[j] << (4 * j);
            hi |= c[8 + j] << (4 * j);
        }
    }
    return make_uint2(lo, hi);
}

}  // namespace reqat
