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

__device__ __forceinline__ void store16(uint16_t *__restrict__ p, const float (&x)[16]) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = bf16_rne_from_float(x[2 * i]) | (bf16_rne_from_float(x[2 * i + 1]) << 16);
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
    int64_t T, ldq, ldk, ldv, ldq_out, rope_len;
    int q_heads;                           // 0: no queries
};

// A thread's item is channels 16 p .. 16 p + 15 and the same of the other half of one head of
// one token; heads count queries, then keys, then values.
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(const AppendArgs a) {
    constexpr int kPairs = D / 32;
    const int heads = a.q_heads + 2 * a.c.heads;
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (item >= a.T * heads * kPairs) return;
    const int p = (int)(item % kPairs);
    const int64_t th = item / kPairs, t = th / heads;
    int h = (int)(th - t * heads);
    const bool is_q = h < a.q_heads;
    h -= is_q ? 0 : a.q_heads;
    const bool is_v = !is_q && h >= a.c.heads;
    h -= is_v ? a.c.heads : 0;
    const int64_t slot = is_q ? 0 : a.slots[t];
    if (slot < 0 || slot >= a.c.slots()) return;           // padding
    const int c0 = 16 * p, c1 = c0 + D / 2;
    const uint16_t *src = (is_q ? a.q + t * a.ldq : is_v ? a.v + t * a.ldv : a.k + t * a.ldk) + h * D;
    float x[2][16];
    load16(src + c0, x[0]);
    load16(src + c1, x[1]);
    if (!is_v && a.cos) {
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
    if (is_q) {
        uint16_t *dst = a.q_out + t * a.ldq_out + h * D;
        store16(dst + c0, x[0]);
        store16(dst + c1, x[1]);
        return;
    }
    const int64_t page = slot >> a.c.page_log2;
    const int tok = (int)(slot & ((int64_t(1) << a.c.page_log2) - 1));
    const int64_t run = a.c.run(page, h);
    const Kv4G G = kv4_make_g(is_v ? *a.c.gv : *a.c.gk);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int b = p + half * (D / 32);
        if (!is_v && a.c.shift) {
            float m[16];
            load_f32x16(a.c.shift + h * D + 16 * b, m);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[half][j] = x[half][j] - m[j];
        }
        const uint32_t am = kv4_block_max(x[half]);
        // values, and keys without rotation and shift, are bfloat16: midpoints are common there
        const bool bf16 = is_v || (!a.cos && !a.c.shift);
        uint2 w;
        uint32_t sbyte;
        if (bf16) {
            const Kv4Rounded R = kv4_round<true>(x[half], am, G);
            w = kv4_codes(x[half], R, G);
            sbyte = R.sbyte;
        } else {
            const Kv4Rounded R = kv4_round<false>(x[half], am, G);
            w = kv4_codes(x[half], R, G);
            sbyte = R.sbyte;
        }
        if (is_v) {
            uint8_t *d = a.c.vc + kv4_v_codes(run, tok, b, D);
            *reinterpret_cast<uint32_t *>(d) = w.x;
            *reinterpret_cast<uint32_t *>(d + 16) = w.y;
            a.c.vs[kv4_v_scales(run, tok, b, D)] = (uint8_t)sbyte;
        } else {
            *reinterpret_cast<uint2 *>(a.c.kc + kv4_k_codes(run, tok, D) + 8 * b) = w;
            a.c.ks[kv4_k_scales(run, tok, D) + b] = (uint8_t)sbyte;
        }
    }
}

// The 16 values of a block as bfloat16: RN(c s g), or RN(RN32(c s g) + shift).  With a
// power-of-two g that keeps s g inside FP32's normal range c s g is exact there; FP64 otherwise.
__device__ __forceinline__ void decode16(uint2 w, uint32_t sbyte, const Kv4G &G, const float *__restrict__ shift,
                                         uint16_t *__restrict__ y) {
    uint32_t o[16];
    float m[16];
    if (shift) load_f32x16(shift, m);
    const bool bad = (sbyte & 0x7Fu) == 0x7Fu;
    const float H = 0.5f * e4m3_value(sbyte) * G.g;
    const bool f32 = G.f32 && (H == 0.0f || H >= 0x1p-126f);
    const double Hd = 0.5 * (double)e4m3_value(sbyte) * G.gd;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint32_t c = ((j < 8 ? w.x : w.y) >> (4 * (j & 7))) & 15u;
        const float mag = (float)(c & 7u);
        const float n = (c & 8u) ? -mag : mag;
        if (shift) {
            const float v = f32 ? n * H : (float)((double)n * Hd);
            o[j] = bf16_rne_from_float(v + m[j]);
        } else {
            o[j] = f32 ? bf16_rne_from_float(n * H) : bf16_rne_from_double((double)n * Hd);
        }
        if (bad) o[j] = 0x7FC0u;
    }
    uint4 *dst = reinterpret_cast<uint4 *>(y);
    dst[0] = make_uint4(o[0] | (o[1] << 16), o[2] | (o[3] << 16), o[4] | (o[5] << 16), o[6] | (o[7] << 16));
    dst[1] = make_uint4(o[8] | (o[9] << 16), o[10] | (o[11] << 16), o[12] | (o[13] << 16), o[14] | (o[15] << 16));
}

// A thread's item is one block of 16 channels of one head of one slot, keys and values.
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_gather_kernel(const Kv4View c, const int64_t *__restrict__ slots, int64_t T,
                                                              uint16_t *__restrict__ ky, int64_t ldk,
                                                              uint16_t *__restrict__ vy, int64_t ldv, bool add_shift) {
    constexpr int kBlocks = D / 16;
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (item >= T * c.heads * kBlocks) return;
    const int b = (int)(item % kBlocks);
    const int64_t th = item / kBlocks, t = th / c.heads;
    const int h = (int)(th - t * c.heads);
    const int64_t slot = slots[t];
    const int64_t at = h * D + 16 * b;
    if (slot < 0 || slot >= c.slots()) {                   // padding
        const uint4 z = make_uint4(0, 0, 0, 0);
        if (ky) reinterpret_cast<uint4 *>(ky + t * ldk + at)[0] = reinterpret_cast<uint4 *>(ky + t * ldk + at)[1] = z;
        if (vy) reinterpret_cast<uint4 *>(vy + t * ldv + at)[0] = reinterpret_cast<uint4 *>(vy + t * ldv + at)[1] = z;
        return;
    }
    const int tok = (int)(slot & ((int64_t(1) << c.page_log2) - 1));
    const int64_t run = c.run(slot >> c.page_log2, h);
    if (ky) {
        const uint2 w = *reinterpret_cast<const uint2 *>(c.kc + kv4_k_codes(run, tok, D) + 8 * b);
        decode16(w, c.ks[kv4_k_scales(run, tok, D) + b], kv4_make_g(*c.gk), add_shift ? c.shift + at : nullptr,
                 ky + t * ldk + at);
    }
    if (vy) {
        const uint8_t *s = c.vc + kv4_v_codes(run, tok, b, D);
        const uint2 w = make_uint2(*reinterpret_cast<const uint32_t *>(s), *reinterpret_cast<const uint32_t *>(s + 16));
        decode16(w, c.vs[kv4_v_scales(run, tok, b, D)], kv4_make_g(*c.gv), nullptr, vy + t * ldv + at);
    }
}

unsigned blocks_for(int64_t items) { return (unsigned)((items + kThreads - 1) / kThreads); }

}  // namespace

hipError_t launch_kv4_append(const Kv4View &c, int64_t T, const int64_t *slots, const uint16_t *k, int64_t ldk,
                             const uint16_t *v, int64_t ldv, const uint16_t *q, int64_t ldq, int q_heads,
                             uint16_t *q_out, int64_t ldq_out, const float *cos, const float *sin,
                             const int32_t *positions, int64_t rope_len, hipStream_t stream) {
    const AppendArgs a = {c, slots, q, k, v, q_out, cos, sin, positions, T, ldq, ldk, ldv, ldq_out, rope_len, q_heads};
    const unsigned n = blocks_for(T * (q_heads + 2 * c.heads) * (c.D / 32));
    if (c.D == 128) kv4_append_kernel<128><<<n, kThreads, 0, stream>>>(a);
    else kv4_append_kernel<64><<<n, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv4_gather(const Kv4View &c, int64_t T, const int64_t *slots, uint16_t *k, int64_t ldk, uint16_t *v,
                             int64_t ldv, bool add_shift, hipStream_t stream) {
    const unsigned n = blocks_for(T * c.heads * (c.D / 16));
    const bool sh = add_shift && c.shift;
    if (c.D == 128) kv4_gather_kernel<128><<<n, kThreads, 0, stream>>>(c, slots, T, k, ldk, v, ldv, sh);
    else kv4_gather_kernel<64><<<n, kThreads, 0, stream>>>(c, slots, T, k, ldk, v, ldv, sh);
    return hipGetLastError();
}

}  // namespace reqat
