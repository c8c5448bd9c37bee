// Writer and reader of the paged 4-bit cache (the KV4 cache of the NVFP4 W4A4KV4 setting,
// Sec. 4.3; layout in kv4_cache.h).
//
// kv4_append_kernel: one pass over the new tokens of the QKV product.  Queries and keys are
// rotated to their positions (halves of a head paired: channel c with c + D/2),
//   lo' = RN(RN(lo cos) - RN(hi sin)),   hi' = RN(RN(hi cos) + RN(lo sin))   (FP32),
// queries rounded to bfloat16, keys less the shift, and keys and values quantized by the rules
// of reqat_quantize_kv4 into their slots.  No intermediate goes through memory.
// kv4_gather_kernel: the values that slots hold, as bfloat16.
#include "internal.h"
#include "kv4_block.h"

namespace reqat {

namespace {

constexpr int kThreads = 256;
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// 16 bfloat16 values as FP32
__device__ __forceinline__ void load16(const uint16_t *__restrict__ p, float (&x)[16]) {
    const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[2 * i] = f32_from_bits(w[i] << 16);
        x[2 * i + 1] = f32_from_bits(w[i] & 0xFFFF0000u);
    }
}

// Two FP32 values rounded to bfloat16 (nearest even).
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const b2 y = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, y);
}

__device__ __forceinline__ void store16(uint16_t *__restrict__ p, const float (&x)[16]) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

__device__ __forceinline__ void load_f32x16(const float *__restrict__ p, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 v = reinterpret_cast<const float4 *>(p)[i];
        x[4 * i] = v.x;
        x[4 * i + 1] = v.y;
        x[4 * i + 2] = v.z;
        x[4 * i + 3] = v.w;
    }
}

struct AppendArgs {
    Kv4View c;
    const int64_t *slots;
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    const float *cos, *sin;                // [rope_len][D / 2], or null: no rotation
    const int32_t *positions;
    int64_t ldq, ldk, ldv, ldq_out, rope_len;
    int T, q_heads;                        // tokens of this launch; 0 heads: no queries
    int kv_blocks;                         // workgroups of the keys, and of the values
};

// Quantizes 16 values into block b of token `tok`.  kBf16: they are bfloat16 numbers, where midpoints are common.
template <int D, bool kValues, bool kBf16>
__device__ __forceinline__ void put_block(const AppendArgs &a, const float (&x)[16], const Kv4G &G, int64_t run, int tok, int b) {
    const Kv4Rounded R = kv4_round<kBf16>(x, kv4_block_max(x), G);
    const uint2 w = kv4_codes(x, R, G);
    if constexpr (kValues) {
        uint8_t *d = a.c.vc + kv4_v_codes(run, tok, b, D);
        *reinterpret_cast<uint32_t *>(d) = w.x;
        *reinterpret_cast<uint32_t *>(d + 16) = w.y;
        a.c.vs[kv4_v_scales(run, tok, b, D)] = (uint8_t)R.sbyte;
    } else {
        *reinterpret_cast<uint2 *>(a.c.kc + kv4_k_codes(run, tok, D) + 8 * b) = w;
        a.c.ks[kv4_k_scales(run, tok, D) + b] = (uint8_t)R.sbyte;
    }
}

// A thread's item is channels 16 p .. 16 p + 15 and the same of the other half of one head of one token.  The first
// workgroups take the keys, the next the values, the last the queries: a wave does one of the three (with heads of
// all kinds in a wave, 5003 tokens of 28 + 4 + 4 heads took 32 us; rounding by bit arithmetic in FP32 was part of that).
// Two 16-byte loads at each half of a head give a lane whole blocks of 16 channels and both members of its pairs.
// Bound by memory: those 5003 tokens move 87 MB in 21.8 us, 4.0 TB/s (a copy: 5.2; waves wait on 0.72 of their cycles, VALU
// issue on 0.38).  64 tokens of 40 + 8 + 8 heads: 5.3 us, a launch and, for a key, five trips to memory in turn, each behind a
// branch: the row, its position, cos and sin, the slot, the scale and the shift.
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(const AppendArgs a) {
    constexpr int kPairs = D / 32;
    const int kind = (int)blockIdx.x < a.kv_blocks ? 0 : (int)blockIdx.x < 2 * a.kv_blocks ? 1 : 2;   // keys, values, queries
    const int heads = kind == 2 ? a.q_heads : a.c.heads;
    const uint32_t item = (blockIdx.x - kind * a.kv_blocks) * kThreads + threadIdx.x;
    const uint32_t th = item / kPairs, t = th / heads;
    if (t >= (uint32_t)a.T) return;
    const int p = (int)(item % kPairs), h = (int)(th - t * heads);
    const int c0 = 16 * p, c1 = c0 + D / 2;
    const uint16_t *src = (kind == 2 ? a.q + t * a.ldq : kind == 1 ? a.v + t * a.ldv : a.k + t * a.ldk) + h * D;
    float x[2][16];
    load16(src + c0, x[0]);
    load16(src + c1, x[1]);
    if (kind != 1 && a.cos) {
        const int64_t pos = a.positions[t];
        if (pos >= 0 && pos < a.rope_len) {
            float c[16], s[16];
            load_f32x16(a.cos + pos * (D / 2) + c0, c);
            load_f32x16(a.sin + pos * (D / 2) + c0, s);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float lo = x[0][j], hi = x[1][j];
                x[0][j] = lo * c[j] - hi * s[j];
                x[1][j] = hi * c[j] + lo * s[j];
            }
        } else {                                           // no such row of the tables
#pragma unroll
            for (int j = 0; j < 16; ++j) x[0][j] = x[1][j] = __builtin_nanf("");
        }
    }
    if (kind == 2) {
        uint16_t *dst = a.q_out + t * a.ldq_out + h * D;
        store16(dst + c0, x[0]);
        store16(dst + c1, x[1]);
        return;
    }
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.c.slots()) return;           // padding
    const int tok = (int)(slot & ((int64_t(1) << a.c.page_log2) - 1));
    const int64_t run = a.c.run(slot >> a.c.page_log2, h);
    if (kind == 1) {
        const Kv4G G = kv4_make_g(*a.c.gv);
        put_block<D, true, true>(a, x[0], G, run, tok, p);
        put_block<D, true, true>(a, x[1], G, run, tok, p + D / 32);
        return;
    }
    const Kv4G G = kv4_make_g(*a.c.gk);
    if (a.c.shift) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float m[16];
            load_f32x16(a.c.shift + h * D + (half ? c1 : c0), m);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[half][j] = x[half][j] - m[j];
        }
    }
    if (a.cos || a.c.shift) {
        put_block<D, false, false>(a, x[0], G, run, tok, p);
        put_block<D, false, false>(a, x[1], G, run, tok, p + D / 32);
    } else {
        put_block<D, false, true>(a, x[0], G, run, tok, p);
        put_block<D, false, true>(a, x[1], G, run, tok, p + D / 32);
    }
}

// The eight values of a dword of codes as bfloat16: RN(c s g), or RN(RN32(c s g) + shift).  With a power-of-two g in the
// range below c s g is exact in FP32: a code's bits in a half word are n 2^-20 as FP16 (sign at bit 15, n at bits 6:4), and
// one mixed FMA per value multiplies them by H 2^20 (H = s g / 2) and adds the shift.  FP64 otherwise.
__device__ __forceinline__ uint4 decode8(uint32_t w, uint32_t sbyte, const Kv4G &G, const float *__restrict__ shift) {
    uint32_t o[4];
    float m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = -0.0f;              // keeps the sign of a zero
    if (shift) {
        const float4 x = reinterpret_cast<const float4 *>(shift)[0], y = reinterpret_cast<const float4 *>(shift)[1];
        m[0] = x.x; m[1] = x.y; m[2] = x.z; m[3] = x.w;
        m[4] = y.x; m[5] = y.y; m[6] = y.z; m[7] = y.w;
    }
    if (G.f32 && G.kg >= -100 && G.kg <= 90) {
        const float up = 0x1p19f * e4m3_value(sbyte) * G.g;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            // bytes 2 k, 2 k + 1: elements 4 k (low nibble), 4 k + 1 (high) and 4 k + 2, 4 k + 3, each byte twice in its half
            const uint32_t b = __builtin_amdgcn_perm(w, w, k ? 0x03030202u : 0x01010000u);
            const h2 lo = __builtin_bit_cast(h2, (b << 4) & 0x80708070u), hi = __builtin_bit_cast(h2, b & 0x80708070u);
            o[2 * k] = bf16_pair(__builtin_fmaf((float)lo[0], up, m[4 * k]), __builtin_fmaf((float)hi[0], up, m[4 * k + 1]));
            o[2 * k + 1] = bf16_pair(__builtin_fmaf((float)lo[1], up, m[4 * k + 2]), __builtin_fmaf((float)hi[1], up, m[4 * k + 3]));
        }
    } else {
        const double H = 0.5 * (double)e4m3_value(sbyte) * G.gd;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t z[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t c = (w >> (4 * (2 * k + e))) & 15u;
                const double v = (c & 8u ? -H : H) * (double)(c & 7u);
                z[e] = shift ? bf16_rne_from_float((float)v + m[2 * k + e]) : bf16_rne_from_double(v);
            }
            o[k] = z[0] | (z[1] << 16);
        }
    }
    const bool bad = (sbyte & 0x7Fu) == 0x7Fu;
    const uint32_t nan = 0x7FC07FC0u;
    return bad ? make_uint4(nan, nan, nan, nan) : make_uint4(o[0], o[1], o[2], o[3]);
}

// 16 bytes written past the L2, which has codes to keep: at 32768 tokens of 8 heads 34.4 us against 45.5, at 2000 tokens
// 5.0 against 5.3 (before each XCD took a run of them).  (For the queries of the append it is no gain: 8000 tokens of 40 + 8 + 8 heads 51 us against 48.)
__device__ __forceinline__ void stream16(uint16_t *__restrict__ p, const uint4 &x) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u4, x), reinterpret_cast<u4 *>(p));
}

// A thread's item is eight channels of one head of one slot, keys and values: a wave writes 1 KB of adjacent bytes
// at a time (with 16 channels a thread and two stores of every other 16 bytes, 32768 tokens of 8 heads took 54 us).
// Workgroups are dealt to the eight XCDs in turn; each XCD takes a contiguous run of items, since four adjacent tokens share
// the 16-byte pieces of their value codes and sixteen a line of their scales, which two and eight XCDs then fetched
// (32768 tokens of 8 heads: 86 MB read for 38, 34.5 us against 31.8; 5003 of 4 heads: 4.5 against 4.1).  172 MB in
// 30.8 us call after call (5.6 TB/s) and 27.1 among other work: bound by memory, where a copy runs at 5.0 to 5.2 TB/s; VALU issue
// takes 0.89 of the SIMD cycles by then.
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_gather_kernel(const Kv4View c, const int64_t *__restrict__ slots, int T,
                                                              uint16_t *__restrict__ ky, int64_t ldk,
                                                              uint16_t *__restrict__ vy, int64_t ldv, bool add_shift) {
    constexpr int kWords = D / 8;
    const uint32_t xcd = blockIdx.x % 8, per = gridDim.x / 8, rem = gridDim.x % 8;
    const uint32_t block = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
    const uint32_t item = block * kThreads + threadIdx.x;
    const uint32_t th = item / kWords, t = th / c.heads;
    if (t >= (uint32_t)T) return;
    const int w = (int)(item % kWords), h = (int)(th - t * c.heads);
    const int64_t slot = slots[t];
    const int64_t at = h * D + 8 * w;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;               // padding: zeros
    if (slot >= 0 && slot < c.slots()) {
        const int tok = (int)(slot & ((int64_t(1) << c.page_log2) - 1));
        const int64_t run = c.run(slot >> c.page_log2, h);
        if (ky) {
            const uint32_t x = *reinterpret_cast<const uint32_t *>(c.kc + kv4_k_codes(run, tok, D) + 4 * w);
            k = decode8(x, c.ks[kv4_k_scales(run, tok, D) + w / 2], kv4_make_g(*c.gk), add_shift ? c.shift + at : nullptr);
        }
        if (vy) {
            const uint32_t x = *reinterpret_cast<const uint32_t *>(c.vc + kv4_v_codes(run, tok, w / 2, D) + 16 * (w & 1));
            v = decode8(x, c.vs[kv4_v_scales(run, tok, w / 2, D)], kv4_make_g(*c.gv), nullptr);
        }
    }
    if (ky) stream16(ky + t * ldk + at, k);
    if (vy) stream16(vy + t * ldv + at, v);
}

// Tokens of one launch: its items (at most 16 a token and head) are numbered in 32 bits.
int64_t slice_of(int heads) { return (int64_t(1) << 27) / heads; }

unsigned blocks_for(int64_t items) { return (unsigned)((items + kThreads - 1) / kThreads); }

}  // namespace

hipError_t launch_kv4_append(const Kv4View &c, int64_t T, const int64_t *slots, const uint16_t *k, int64_t ldk,
                             const uint16_t *v, int64_t ldv, const uint16_t *q, int64_t ldq, int q_heads,
                             uint16_t *q_out, int64_t ldq_out, const float *cos, const float *sin,
                             const int32_t *positions, int64_t rope_len, hipStream_t stream) {
    const int64_t slice = slice_of(c.heads > q_heads ? c.heads : q_heads);
    for (int64_t t = 0; t < T; t += slice) {
        const int n = (int)(T - t < slice ? T - t : slice);
        const int kv_blocks = (int)blocks_for((int64_t)n * c.heads * (c.D / 32));
        const AppendArgs a = {c, slots + t, q_heads ? q + t * ldq : q, k + t * ldk, v + t * ldv,
                              q_heads ? q_out + t * ldq_out : q_out, cos, sin, positions ? positions + t : positions,
                              ldq, ldk, ldv, ldq_out, rope_len, n, q_heads, kv_blocks};
        const unsigned grid = 2 * kv_blocks + blocks_for((int64_t)n * q_heads * (c.D / 32));
        if (c.D == 128) kv4_append_kernel<128><<<grid, kThreads, 0, stream>>>(a);
        else kv4_append_kernel<64><<<grid, kThreads, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kv4_gather(const Kv4View &c, int64_t T, const int64_t *slots, uint16_t *k, int64_t ldk, uint16_t *v,
                             int64_t ldv, bool add_shift, hipStream_t stream) {
    const int64_t slice = slice_of(c.heads);
    const bool sh = add_shift && c.shift;
    for (int64_t t = 0; t < T; t += slice) {
        const int n = (int)(T - t < slice ? T - t : slice);
        const unsigned grid = blocks_for((int64_t)n * c.heads * (c.D / 8));
        uint16_t *kt = k ? k + t * ldk : k, *vt = v ? v + t * ldv : v;
        if (c.D == 128) kv4_gather_kernel<128><<<grid, kThreads, 0, stream>>>(c, slots + t, n, kt, ldk, vt, ldv, sh);
        else kv4_gather_kernel<64><<<grid, kThreads, 0, stream>>>(c, slots + t, n, kt, ldk, vt, ldv, sh);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace reqat
