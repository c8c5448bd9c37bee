// Attention over the paged 4-bit cache (W4A4KV4 serving, Sec. 4.3; layout in kv4_cache.h):
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j - m_i),  j over the row's visible tokens.
// The shift of the keys is left out of the scores: q . m is the same for every key of a row,
// and a softmax does not change when its scores all move by as much.
//
// Arithmetic.  A code times its block scale has at most 7 significant bits, so keys and values are exact
// in FP16: a code's half word, sign at bit 15 and magnitude n at bits 6:4, is n 2^-20; the E4M3 scale
// enters as s 2^7 (<= 57344), and the product n s 2^-13 is a multiple of 2^-22.  A query row takes a
// power-of-two factor that puts its largest value into [2^14, 2^15), so that its bfloat16 values are FP16
// numbers (those below 2^-28 of the largest are rounded, to 2^-39 of it).  The scores sum in FP32.  Weights p =
// 2^(s - r) are rounded to FP16 (11 bits, 3 more than the output has): r trails the running maximum,
// at least 7 and at most 15 below it, so p is at most 2^15 and the FP16 range reaches 2^-31 of the largest
// weight or below; the sum of weights is taken in FP32 before that rounding.  In a row whose largest exponent passes 2^24,
// where FP32 has no number 7 below it, weights count from the score itself: Reference.
#include <type_traits>

#include "fp4_device.h"
#include "g2l.h"
#include "internal.h"
#include "kv4_queue.h"

namespace reqat {

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

typedef const __attribute__((address_space(4))) int *ConstInt;

constexpr uint32_t kCodeMask = 0x80708070u;    // sign and magnitude of a code in either half word
constexpr float kScaleUp = 128.0f;             // FP16 scales are s 2^7
constexpr float kBelow = 7.0f;                 // r = maximum - kBelow when it is renewed
constexpr float kMostSum = 32768.0f;           // ... which it is when a lane's weights of a step sum to more: none is above
constexpr float kMostLarge = 11.0f;            // and when an exponent of a large score's row is above this: the sum of 16 stays below
constexpr float kLargeScore = 0x1p24f;         // exponents from which a reference is a score
constexpr float kHugeFactor = 0x1p100f;        // factors from which an exponent may pass the FP32 range (scores stay below 2^21)
constexpr double kNoPiece = -0x1p1000;         // below every reference
constexpr int kNoToken = 0x7FFFFFFF;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

__device__ __forceinline__ uint32_t scaled(uint32_t code_bits, h2 s) {
    return __builtin_bit_cast(uint32_t, (h2)(__builtin_bit_cast(h2, code_bits) * s));
}

__device__ __forceinline__ h8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(h8, make_uint4(a, b, c, d));
}

// Maximum (sum) over the four lanes that share lane % 16.
__device__ __forceinline__ float max16(float x) {
    x = __builtin_fmaxf(x, __shfl_xor(x, 16, 64));
    return __builtin_fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float sum16(float x) {
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Largest magnitude pattern of 8 N bfloat16 values, in both halves' maximum (a non-finite one: 0x7F80 or above).
template <int N> __device__ __forceinline__ uint32_t largest(const uint4 (&w)[N]) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[e] & 0x7FFF7FFFu));
    }
    return m[0] > m[1] ? m[0] : m[1];
}

// The exponent that takes a row whose largest pattern is `top` to [2^14, 2^15) (a row with a NaN or Inf stays one).
__device__ __forceinline__ int row_shift(uint32_t top) {
    return top == 0u || top >= 0x7F80u ? 0 : 15 - __builtin_amdgcn_frexp_expf(f32_from_bits(top << 16));
}

// Eight bfloat16 values times 2^shift as FP16, in the order that a dword of codes is unpacked in: 0 2 1 3 4 6 5 7.
__device__ __forceinline__ h8 query_f16(const uint4 &w, int shift) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    _Float16 y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        y[e] = (_Float16)__builtin_ldexpf(f32_from_bits((e & 1) ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16), shift);
    return h8{y[0], y[2], y[1], y[3], y[4], y[6], y[5], y[7]};
}

// From scores of such a row to exponents of two.  A code is half its integer: 2^-13 n s = 2^-12 (n / 2) s.
// Finite, since a score minus itself is multiplied by it: at the bound any two scores are still worlds apart.
// Exponents apart: the scales' product may leave the FP32 range where the factor does not.
__device__ __forceinline__ float score_factor(const Kv4AttnArgs &a, int shift) {
    const float g = *a.c.gk;
    const float c = __builtin_ldexpf(__builtin_amdgcn_frexp_mantf(a.scale) * kLog2e * __builtin_amdgcn_frexp_mantf(g),
                                     __builtin_amdgcn_frexp_expf(a.scale) + __builtin_amdgcn_frexp_expf(g) + 12 - shift);
    return __builtin_fminf(__builtin_fmaxf(c, 0x1p-126f), 0x1p127f);
}

// What a row's weights p = 2^(s c - r) are taken from.  r = RN(RN(s' c) - 7), s' the highest score when it was renewed,
// as long as that leaves r well-defined.  From exponents of 2^24 on the step from one FP32 number to the next swallows
// the 7 (and later the FP16 range): then p = 2^((s - s') c + 7), exact near s', and r is NaN, whose sums send every
// step of such a row to the branch that takes this form.  FP64 holds s' c - 7 of both kinds for joining.
struct Reference {
    float r, score;

    __device__ __forceinline__ bool large() const { return r != r; }
    __device__ __forceinline__ void none(float c) {                      // below every score
        r = c < kHugeFactor ? kLowest : __builtin_nanf("");
        score = kLowest;
    }
    // From the highest score and the sum of a step's weights, in the first form: whether they are too large for it.
    __device__ __forceinline__ bool outgrown(float top, float c, float total) const {
        return large() ? __builtin_fmaf(top - score, c, kBelow) > kMostLarge : total > kMostSum;
    }
    // Renewed for `top`; returns what weights so far change by.
    __device__ __forceinline__ float renew(float top, float c) {
        const float t = top * c, next = c < kHugeFactor && __builtin_fabsf(t) < kLargeScore ? t - kBelow : __builtin_nanf("");
        const bool next_large = next != next;
        const float x = large() ? (next_large ? (score - top) * c : __builtin_fmaf(score, c, -next) - kBelow)
                                : (next_large ? __builtin_fmaf(-top, c, r) + kBelow : r - next);
        r = next;
        score = top;
        return __builtin_amdgcn_exp2f(x);
    }
    __device__ __forceinline__ float weight(float s, float c) const {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(s - (large() ? score : 0.0f), c, large() ? kBelow : -r));
    }
    __device__ __forceinline__ double at(float c) const { return large() ? (double)score * c - kBelow : (double)r; }
};

__device__ __forceinline__ float exp2_of(double below) { return __builtin_amdgcn_exp2f((float)below); }

__device__ __forceinline__ float log_sum(double at, float sum) {
    return (float)((at + (double)__builtin_log2f(sum)) * kLn2);
}

// What a row's sum of weights and values is multiplied by; the scale of the values comes last, so that it alone can
// leave the FP32 range, as the values then do.
__device__ __forceinline__ float finish_factor(bool lost, bool none, float sum) {
    return lost ? __builtin_nanf("") : none ? 0.0f : 4096.0f / sum;
}

// A row's share of a call that is cut into pieces, beside its unfinished output: reference and sum of weights.
struct __attribute__((aligned(16))) PieceRow {
    double at;
    float sum, unused;
};

// The queries and tokens of sequence b.
struct Seq {
    int64_t q0;          // first query row
    int nq;              // queries
    int len;             // cached tokens
    bool lost;           // more tokens than the caller's bounds or the table hold: NaN
};

__device__ __forceinline__ Seq sequence(const Kv4AttnArgs &a, int b) {
    Seq s;
    int64_t q0 = b, q1 = b + 1;
    if (a.q_start) {
        q0 = a.q_start[b];
        q1 = a.q_start[b + 1];
        q0 = q0 < 0 ? 0 : q0;
        q1 = q1 > a.T ? a.T : q1;
    }
    s.q0 = q0;
    s.nq = (int)(q1 > q0 ? q1 - q0 : 0);
    s.len = a.kv_len[b] < 0 ? 0 : a.kv_len[b];
    s.lost = s.len > a.max_kv || s.len > (a.table_cols << a.c.page_log2) || (s.len > 0 && a.c.pages == 0);
    return s;
}

// Tokens that query i of the sequence sees: 0 .. visible - 1.
__device__ __forceinline__ int visible(const Kv4AttnArgs &a, const Seq &s, int i) {
    const int n = a.causal ? s.len - s.nq + i + 1 : s.len;
    return n < 0 ? 0 : n;
}

// ------------------------------------------------------------------ few queries

// A wave takes 32 tokens a step against 16 NT rows (query, head of the KV head's group), alone: codes go
// from memory to registers in the matrix cores' operand layout, and nothing is shared until the end.
//   S^T = K Q^T  (16 tokens x 16 rows, K = 32 channels): lane (r, g) = (lane % 16, lane / 16) holds token r, channels
//     D/4 g ..; it gets the scores of row r and tokens 4 g .. 4 g + 3, twice.
//   O^T = V^T P^T (16 channels x 16 rows, K = 32 tokens): those eight tokens are its share of the K axis, so the weights
//     are the operand as they stand, and the cache holds the values of four tokens together.  Tile c has channels
//     8 w + c of the dwords w.
// The operands are this way round so that scores and weights stay in their lanes: no transpose, no LDS.  With 16 rows
// to a tile and 5 to 8 heads a group the matrix cores do two to three times the work there is, and have time for it.
//
// Bound by memory where the call is large, with the VALU's unpacking not far behind it: 728 MB (64 sequences
// of up to 16384 tokens, 8 KV heads of 128) in 137 to 140 us, 5.3 TB/s with the join's 6 us, reads alone running at 6.0 to
// 6.4; counters: VALU issue on 0.75 of the SIMD cycles, matrix pipe busy on 0.15.  131072 tokens of one sequence: 151 MB in
// 34.9 us, 29 without the join.  Below some 50 MB by the steps in a row: first codes, queries, the join of the waves, then
// the other launch (1021 tokens of 2 heads: 8.7 us, 7.1 and 2.9 by kernel).  Up to 32 rows (25: 52 MB in 27.8 us) twice the
// products and exponentials stand beside the same codes.  Heads of 64: half the bytes, and the same steps, whose loads fetch
// every operand twice (lanes g and g + 2 the same keys, r and r + 8 the same values): the full batch 88.8 us, 4.1 TB/s.
template <int D> struct Step {
    uint32_t k[2][D / 32], ks[2];
    uint32_t v[2][4], vs[2];
};

template <int D, int NT, int W>
__global__ __launch_bounds__(64 * W, 2) void kv4_decode_kernel(const Kv4AttnArgs a, int splits, int chunk) {
    using Queue = Kv4Queue;
    constexpr int KW = D / 32, VT = D / 16;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // heads first: workgroups go round the eight XCDs, and an XCD that got the same piece of every sequence would have
    // the last ones empty where lengths differ (64 sequences of up to 16384 tokens, pieces of 2048: 192 us against 165, when
    // it was changed)
    int id = blockIdx.x;
    const int h = id % a.c.heads;
    id /= a.c.heads;
    const int split = id % splits, b = id / splits;
    const int group = a.q_heads / a.c.heads;
    const int t0 = split * chunk;

    const ConstInt table = (ConstInt)(uintptr_t)(a.table + (int64_t)b * a.ld_table);   // scalar loads
    const int plog = a.c.page_log2, pmask = (1 << plog) - 1, last_entry = (int)a.table_cols - 1;
    constexpr int kStride = 32 * W;
    int t = t0 + 32 * wave;
    // page entries of the first steps, beside the lengths that say whether they are needed
    auto pages = [&](int t, int (&p)[2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = (t + 16 * u) >> plog;
            p[u] = table[at < last_entry ? at : last_entry];
        }
    };
    int p[Queue::kDepth + 1][2] = {};
    if (last_entry >= 0) {
#pragma unroll
        for (int k = 0; k <= Queue::kDepth; ++k) pages(t + k * kStride, p[k]);
    }

    const Seq sq = sequence(a, b);
    const int nq = sq.nq < a.max_q ? sq.nq : (int)a.max_q;
    const int rows = nq * group;                                         // at most 16 NT
    if (rows == 0) return;
    const int see_least = visible(a, sq, 0);
    const int t1 = sq.lost ? 0 : sq.len - t0 < chunk ? sq.len : t0 + chunk;  // this workgroup's tokens
    if (split > 0 && t0 >= t1) return;                                   // the join does not read it

    const uint32_t w_at = D == 128 ? r : r & 7;                        // the lane's dword of value codes
    const uint32_t v_at = g * (2 * D) + w_at * 16, vs_at = g * (D / 4) + (w_at >> 1) * 4;
    // keys: 16 bytes and a dword of scales hold what the lane needs (D = 64: half of the 16 bytes, and lanes 32 .. load
    // what the lower ones do)
    const uint32_t k_at = D == 128 ? r * 64 + g * 16 : r * 32 + (g & 1) * 16, ks_at = D == 128 ? r * 8 + (g >> 1) * 4 : r * 4;
    const uint32_t k_read = D == 128 ? lane * 16 : (r + 16 * (g >> 1)) * 16 + (g & 1) * 8;
    const uint32_t ks_shift = D == 128 ? 16 * (g & 1) : 8 * g;
    // D = 64: sixteen rows of a tile are eight dwords times two: lanes 8 .. 15 take the dword's upper channels
    const uint32_t half = D == 128 ? 0u : (uint32_t)(r >> 3) * 0x02020202u;
    int bad_at = kNoToken;               // the first token, some rows not seeing it, whose values in the lane's block are NaN

    constexpr int kLd = D + 4;
    constexpr int kParts = W < 2 ? W : 2;                                // waves whose rows are in LDS at once
    constexpr int kQueue = W * Queue::kDepth * Queue::kStage, kPart = kParts * 16 * kLd * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kQueue > kPart ? kQueue : kPart];
    uint8_t *queue = lds + wave * (Queue::kDepth * Queue::kStage);
    uint32_t in_bits = 0;                // two for each step on its way, the newest lowest: its pages lie in the cache
    auto issue = [&](int t, const int (&p)[2], uint8_t *stage) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool in = p[u] >= 0 && p[u] < a.c.pages;             // uniform
            in_bits = in_bits << 1 | (in ? 1u : 0u);
            const int tok = (t + 16 * u) & pmask;
            const int64_t run = a.c.run(in ? p[u] : 0, h) + tok;      // tokens (values: a multiple of 4 of them)
            Queue::put(a.c.kc + run * (D / 2), k_at, a.c.vc + run * (D / 2), v_at, a.c.ks + run * (D / 16), ks_at,
                       a.c.vs + run * (D / 16), vs_at, stage, u);
        }
    };
    auto take = [&](const uint8_t *stage, uint32_t bits, Step<D> &st) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (D == 128) {
                const uint4 x = *reinterpret_cast<const uint4 *>(stage + Queue::kKeys + u * 1024 + k_read);
                st.k[u][0] = x.x;
                st.k[u][1] = x.y;
                st.k[u][2] = x.z;
                st.k[u][3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(stage + Queue::kKeys + u * 1024 + k_read);
                st.k[u][0] = x.x;
                st.k[u][1] = x.y;
            }
            const uint4 y = *reinterpret_cast<const uint4 *>(stage + Queue::kValues + u * 1024 + lane * 16);
            st.v[u][0] = y.x;
            st.v[u][1] = y.y;
            st.v[u][2] = y.z;
            st.v[u][3] = y.w;
            st.ks[u] = *reinterpret_cast<const uint32_t *>(stage + Queue::kKeyScales + u * 256 + lane * 4) >> ks_shift;
            st.vs[u] = *reinterpret_cast<const uint32_t *>(stage + Queue::kValueScales + u * 256 + lane * 4);
            if (!(bits >> (1 - u) & 1u)) {                             // uniform: scores NaN, values zero
                st.ks[u] = 0x7F7Fu;
                st.vs[u] = 0u;
            }
        }
    };
    int ahead = 0;                       // steps on their way
#pragma unroll
    for (int k = 0; k < Queue::kDepth; ++k)
        if (t + k * kStride < t1) {
            issue(t + k * kStride, p[k], queue + k * Queue::kStage);
            ++ahead;
        }
    int (&p_next)[2] = p[Queue::kDepth];

    // queries (rows beyond the last repeat the first), the factor from scores to exponents, and what each row sees
    h8 qf[NT][KW];
    float c[NT], sum[NT];
    Reference ref[NT];
    int see[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = 16 * n + r < rows ? 16 * n + r : 0, i = row / group;
        see[n] = 16 * n + r < rows ? visible(a, sq, i) : 0;
        const uint16_t *src = a.q + (sq.q0 + i) * a.ldq + (int64_t)(h * group + row - i * group) * D + (D / 4) * g;
        uint4 w[KW];
#pragma unroll
        for (int j = 0; j < KW; ++j) w[j] = reinterpret_cast<const uint4 *>(src)[j];
        uint32_t top = largest(w);
        uint32_t x = __shfl_xor(top, 16, 64);
        top = top > x ? top : x;
        x = __shfl_xor(top, 32, 64);
        const int shift = row_shift(top > x ? top : x);
#pragma unroll
        for (int j = 0; j < KW; ++j) qf[n][j] = query_f16(w[j], shift);
        c[n] = score_factor(a, shift);
        ref[n].none(c[n]);
        sum[n] = 0.0f;
    }
    f32x4 o[VT][NT];
#pragma unroll
    for (int x = 0; x < VT; ++x)
#pragma unroll
        for (int n = 0; n < NT; ++n) o[x][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto compute = [&](int t, Step<D> &st) {
        f32x4 s[2][NT];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const h2 sc = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(st.ks[u], kScaleUp, false);
            const h2 sc0 = {sc[0], sc[0]}, sc1 = {sc[1], sc[1]};
#pragma unroll
            for (int n = 0; n < NT; ++n) s[u][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < KW; ++j) {
                const h2 sj = j < 2 ? sc0 : sc1;
                const uint32_t x = __builtin_amdgcn_perm(st.k[u][j], st.k[u][j], 0x01010000u);
                const uint32_t y = __builtin_amdgcn_perm(st.k[u][j], st.k[u][j], 0x03030202u);
                const h8 kf = frag(scaled((x << 4) & kCodeMask, sj), scaled(x & kCodeMask, sj),
                                   scaled((y << 4) & kCodeMask, sj), scaled(y & kCodeMask, sj));
#pragma unroll
                for (int n = 0; n < NT; ++n) s[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[n][j], s[u][n], 0, 0, 0);
            }
        }
        const bool edge = t + 32 > see_least;                          // uniform
        if (edge) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (t + 16 * u + 4 * g + i >= see[n]) s[u][n][i] = -__builtin_inff();
            // a hidden value must not reach a row: 0 NaN is NaN.  Beyond every row a scale becomes 0, and so does a
            // NaN scale, whose NaN is put back at the end into the rows that see it.
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = t + 16 * u + 4 * g + i;
                    const bool nan = ((st.vs[u] >> (8 * i)) & 0x7Fu) == 0x7Fu;
                    if (at >= t1 || nan) st.vs[u] &= ~(0xFFu << (8 * i));
                    if (at < t1 && nan) bad_at = bad_at < at ? bad_at : at;
                }
        }
        uint32_t p[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float e[8], total = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 2][n][i & 3], c[n], -ref[n].r));
                total += e[i];
            }
            if (__any(!(total <= kMostSum))) {                           // or NaN: large scores, and what is NaN in earnest
                float top = s[0][n][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = __builtin_fmaxf(top, s[i >> 2][n][i & 3]);
                top = max16(top);
                float f = 1.0f;
                if (ref[n].outgrown(top, c[n], max16(total))) f = ref[n].renew(top, c[n]);   // by the row's own scores alone
                sum[n] *= f;
#pragma unroll
                for (int x = 0; x < VT; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[x][n][i] *= f;
                total = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    e[i] = ref[n].weight(s[i >> 2][n][i & 3], c[n]);
                    total += e[i];
                }
            }
            sum[n] += total;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const h2 z = {(_Float16)e[2 * i], (_Float16)e[2 * i + 1]};
                p[n][i] = __builtin_bit_cast(uint32_t, z);
            }
        }
        h2 sv[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sv[u][0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(st.vs[u], kScaleUp, false);
            sv[u][1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(st.vs[u], kScaleUp, true);
        }
#pragma unroll
        for (int j = 0; j < VT / 2; ++j) {
            uint32_t x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = __builtin_amdgcn_perm(st.v[i >> 1][2 * (i & 1) + 1], st.v[i >> 1][2 * (i & 1)],
                                             0x04040000u + 0x01010101u * j + half);
            const h8 even = frag(scaled((x[0] << 4) & kCodeMask, sv[0][0]), scaled((x[1] << 4) & kCodeMask, sv[0][1]),
                                 scaled((x[2] << 4) & kCodeMask, sv[1][0]), scaled((x[3] << 4) & kCodeMask, sv[1][1]));
            const h8 odd = frag(scaled(x[0] & kCodeMask, sv[0][0]), scaled(x[1] & kCodeMask, sv[0][1]),
                                scaled(x[2] & kCodeMask, sv[1][0]), scaled(x[3] & kCodeMask, sv[1][1]));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const h8 pf = frag(p[n][0], p[n][1], p[n][2], p[n][3]);
                o[2 * j][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, pf, o[2 * j][n], 0, 0, 0);
                o[2 * j + 1][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, pf, o[2 * j + 1][n], 0, 0, 0);
            }
        }
    };

    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    for (uint8_t *stage = queue; t < t1; t += kStride) {
        if (ahead == Queue::kDepth) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Queue::kLoads * (Queue::kDepth - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        Step<D> st;
        take(stage, in_bits >> (2 * (ahead - 1)), st);
        __builtin_amdgcn_s_waitcnt(0xC07F);                              // lgkmcnt(0): the stage is free
        asm volatile("" ::: "memory");
        const int later = t + Queue::kDepth * kStride;
        if (later < t1) issue(later, p_next, stage);
        else --ahead;
        pages(later + kStride, p_next);
        stage = stage == queue + (Queue::kDepth - 1) * Queue::kStage ? queue : stage + Queue::kStage;
        compute(t, st);
    }

    if (__any(bad_at != kNoToken)) {
        // over all tokens of the block; lane (r, g) holds channels of the dwords 4 g .. 4 g + 3.  What a row
        // sees is a prefix: it sees a NaN if it sees the first.
        int x = __shfl_xor(bad_at, 16, 64);
        bad_at = bad_at < x ? bad_at : x;
        x = __shfl_xor(bad_at, 32, 64);
        bad_at = bad_at < x ? bad_at : x;
        const int first = __shfl(bad_at, 4 * g, 64), second = __shfl(bad_at, 4 * g + 2, 64);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int x = 0; x < VT; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((i < 2 ? first : second) < see[n]) o[x][n][i] = __builtin_nanf("");
    }

    // Join the waves: references and sums first, then the rows through LDS.  `finish` turns a row's joined sum into
    // its output; a split leaves its rows as they are, with their reference and sum of weights beside them.
    float (*part)[16][kLd] = reinterpret_cast<float (*)[16][kLd]>(lds);
    __shared__ double refs[W][16 * NT];
    __shared__ float sums[W][16 * NT], finish[16 * NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        sum[n] = sum16(sum[n]);
        if (g == 0) {
            refs[wave][16 * n + r] = ref[n].at(c[n]);
            sums[wave][16 * n + r] = sum[n];
        }
    }
    __syncthreads();
    float *po = reinterpret_cast<float *>(a.workspace);
    const int64_t all = a.B * a.max_q * a.q_heads, first = (int64_t)b * a.max_q;   // partial rows go by sequence, max_q to each
    if ((int)threadIdx.x < rows) {
        const int row = threadIdx.x, i = row / group;
        const int hq = h * group + (row - i * group);
        double top = refs[0][threadIdx.x];
        float total = 0.0f;
#pragma unroll
        for (int w = 1; w < W; ++w) top = __builtin_fmax(top, refs[w][threadIdx.x]);
#pragma unroll
        for (int w = 0; w < W; ++w)
            total = __builtin_fmaf(sums[w][threadIdx.x], exp2_of(refs[w][threadIdx.x] - top), total);
        if (splits > 1) {
            reinterpret_cast<PieceRow *>(po + (int64_t)splits * all * D)[split * all + (first + i) * a.q_heads + hq] = {top, total, 0.0f};
        } else {
            const bool none = visible(a, sq, i) == 0 && !sq.lost;
            finish[threadIdx.x] = finish_factor(sq.lost, none, total);
            if (a.lse) a.lse[(sq.q0 + i) * a.q_heads + hq] = sq.lost ? __builtin_nanf("") : none ? -__builtin_inff() : log_sum(top, total);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        double m = refs[0][16 * n + r];
#pragma unroll
        for (int w = 1; w < W; ++w) m = __builtin_fmax(m, refs[w][16 * n + r]);
        const float f = exp2_of(ref[n].at(c[n]) - m);
        if (n > 0) __syncthreads();
        auto at = [&](int x, int i) -> float & {
            const int rho = 4 * g + i;
            return part[wave % kParts][r][D == 128 ? 8 * rho + x : 8 * (rho & 7) + 4 * (rho >> 3) + x];
        };
#pragma unroll
        for (int round = W / kParts - 1; round >= 0; --round) {          // the later waves' rows first, the earlier add theirs
            if (wave / kParts == round) {
#pragma unroll
                for (int x = 0; x < VT; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i) at(x, i) = round == W / kParts - 1 ? o[x][n][i] * f : __builtin_fmaf(o[x][n][i], f, at(x, i));
            }
            __syncthreads();
        }
        const int have = rows - 16 * n;
        for (int x = threadIdx.x; x < (have < 16 ? have : 16) * (D / 2); x += 64 * W) {
            const int rr = x / (D / 2), ch = x % (D / 2) * 2;
            float y0 = 0.0f, y1 = 0.0f;
#pragma unroll
            for (int w = 0; w < kParts; ++w) {
                y0 += part[w][rr][ch];
                y1 += part[w][rr][ch + 1];
            }
            const int row = 16 * n + rr, i = row / group, hq = h * group + (row - i * group);
            if (splits > 1) {
                *reinterpret_cast<float2 *>(po + (split * all + (first + i) * a.q_heads + hq) * D + ch) = make_float2(y0, y1);
            } else {
                const float f1 = finish[16 * n + rr], g1 = *a.c.gv;
                *reinterpret_cast<uint32_t *>(a.out + (sq.q0 + i) * a.ldo + (int64_t)hq * D + ch) =
                    bf16_rne_from_float(y0 * f1 * g1) | (bf16_rne_from_float(y1 * f1 * g1) << 16);
            }
        }
    }
}

// ------------------------------------------------------------------ prompts

// A workgroup of eight waves takes 256 rows, 32 a wave, and 64 tokens a step.  The codes of a step become FP16
// once, in LDS, in the order of the matrix cores' operands (four waves the keys, four the values, two steps ahead;
// their codes are loaded three steps ahead), and every wave reads them from there:
//   S^T = K Q^T  (32 tokens x 32 rows, K = 16 channels): lane (c, u) = (lane % 32, lane / 32) gets the scores of row c
//     and tokens 8 x + 4 u .. 8 x + 4 u + 3.
//   O^T = V^T P^T (32 channels x 32 rows, K = 16 tokens): eight of those, two groups of four, are its K share.
// The scores of 32 tokens are computed beside the weights of the 32 before.
//
// 256 rows to a workgroup, since unpacking a token costs the same for any number of rows; 32 x 32 products, since each
// operand read feeds twice the work of a 16 x 16 one.  Bound by issue and by power: 8192 queries of 8192 tokens, 40 + 8 heads
// of 128 (687 GFLOP of visible pairs) in 642 to 659 us, 1.04 to 1.07 PFLOP/s (a large library FP16 product, both operands
// along K: 1.39 to 1.49 by the box, its operands being FP16 in memory; MFMA with the operand read
// and the exponential beside it and nothing else: 1.33, at a clock that power holds near 1.56 GHz); counters: matrix
// pipe busy on 0.54 of the cycles, 7.8 VALU instructions to an MFMA (with it), of which unpacking and weights.
// 5 sequences of up to 777 queries and 9001 tokens, 28 + 4 heads: 240 GFLOP in 262 us, 0.92 PFLOP/s, 440 workgroups of unequal
// length on 256 CUs.  Heads of 64 (half the operands, as many exponentials): the prompt in 448 us, 0.77 PFLOP/s.
template <int D> struct Prompt {
    static constexpr int F = D / 16;                     // operands of 1 KB: of 32 tokens' keys; of their values
    static constexpr int kSub = 2 * F * 1024;            // 32 tokens: keys, then values
    static constexpr int kStage = 2 * kSub;
    static constexpr int kRing = 4;
    static constexpr int kOut = 8 * 32 * (D + 1) * 4;         // the rows on their way out
    static constexpr int kLds = kRing * kStage > kOut ? kRing * kStage : kOut;
};

// The sequence with the place-th longest cache (of equal ones the first): what is left to the last workgroups is short.
// Of up to 64 sequences; more are taken as they come.  Uniform.
__device__ __forceinline__ int longest(const Kv4AttnArgs &a, int place) {
    if (a.B == 1 || a.B > 64) return place;
    const int lane = threadIdx.x & 63, mine = lane < a.B ? a.kv_len[lane] : 0;
    int before = 0;
    for (int i = 0; i < (int)a.B; ++i) {
        const int other = __builtin_amdgcn_readlane(mine, i);
        before += other > mine || (other == mine && i < lane) ? 1 : 0;
    }
    return __builtin_ctzll(__ballot(lane < a.B && before == place));
}

template <int D>
__global__ __launch_bounds__(512, 2) void kv4_prompt_kernel(const Kv4AttnArgs a, int qtiles, int splits, int chunk) {
    using C = Prompt<D>;
    constexpr int VT = D / 32, WD = D / 8, CPT = 32 / WD, kRows = 256;
    extern __shared__ __attribute__((aligned(16))) uint8_t ring[];
    __shared__ int bad[D / 16];
    const int lane = threadIdx.x & 63, col = lane & 31, up = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int id = blockIdx.x;
    const int h = id % a.c.heads;
    id /= a.c.heads;
    const int split = id % splits;
    id /= splits;
    const int qt = qtiles - 1 - id % qtiles;                            // the longest rows first,
    const int b = longest(a, id / qtiles);                              // of the longest sequence first
    const int group = a.q_heads / a.c.heads;

    const Seq sq = sequence(a, b);
    const int nq = sq.nq < a.max_q ? sq.nq : (int)a.max_q;
    const int rows = nq * group, row0 = qt * kRows;
    if (row0 >= rows) return;
    const int row_last = row0 + kRows < rows ? row0 + kRows - 1 : rows - 1;
    const int see_least = visible(a, sq, row0 / group), see_most = visible(a, sq, row_last / group);
    const int t0 = split * chunk;
    const int t1 = sq.lost ? 0 : see_most < t0 + chunk ? see_most : t0 + chunk;
    if (split > 0 && t0 >= t1) return;

    const int row = row0 + 32 * wave + col;                             // this lane's row
    const bool there = row < rows;
    const int qi = there ? row / group : 0;
    const int hq = h * group + (there ? row - qi * group : 0);           // rows beyond the last repeat the first
    const int see = there ? visible(a, sq, qi) : 0;
    const int wsee_least = row0 + 32 * wave < rows ? visible(a, sq, (row0 + 32 * wave) / group) : 0;

    f32x16 o[VT];
#pragma unroll
    for (int x = 0; x < VT; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[x][v] = 0.0f;

    // this thread's part of the codes, 16 tokens a wave: keys (waves 0 .. 3) D / 4 channels of a token, values
    // (4 .. 7) eight channels of four tokens
    const bool keys = wave < 4;
    const int my_tok = keys ? lane >> 2 : (lane / WD) * 4, my_at = keys ? lane & 3 : lane % WD;
    const bool has = keys || lane < 4 * WD;
    const int *table = a.table + (int64_t)b * a.ld_table;
    const int plog = a.c.page_log2, pmask = (1 << plog) - 1;
    const uint32_t code_at = my_tok * (D / 2) + my_at * (keys ? D / 8 : 16);
    const uint32_t scale_at = my_tok * (D / 16) + (keys ? my_at * (D / 64) : (my_at >> 1) * 4);
    const uint8_t *codes = keys ? a.c.kc : a.c.vc, *scales = keys ? a.c.ks : a.c.vs;
    // where its operands go.  Keys: dwords my_at (D / 32) + j of token my_tok; a quarter's operands have their lanes turned
    // by 2 my_at, so that eight lanes of a write (two tokens) fall on all banks.  Values: tokens my_tok .. my_tok + 3 and + 8 ..
    // are one operand row: lanes a half (D = 64: a quarter) wave apart swap, the lower ones keep the dword's channels 0 .. 3,
    // the upper ones 4 .. 7.
    const int half = D == 128 ? lane >> 5 : (lane >> 4) & 1, odd = D == 128 ? (lane >> 4) & 1 : (lane >> 3) & 1;
    const uint32_t put_at = ((wave & 3) >> 1) * C::kSub +
                            (keys ? my_at * (D / 64) * 1024 + (((16 * (wave & 1) + my_tok) ^ (2 * my_at)) * 16)
                                  : (C::F + (wave & 1)) * 1024 + (my_at + 32 * odd) * 16 + half * (4 / CPT) * 2048);
    uint32_t turned[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) turned[j] = (lane ^ (2 * j)) * 16;
    if (threadIdx.x < D / 16) bad[threadIdx.x] = kNoToken;

    struct Codes {
        uint32_t w[4], s;
        bool in;                         // the page lies in the cache (looked at when the loads have long been issued)
    };
    auto page_of = [&](int t) {
        // a vector load: a scalar one would share the counter that the operand reads are waited for with
        const int tt = t + 16 * (wave & 3);
        int at = tt < t1 ? tt >> plog : 0;
        asm volatile("" : "+v"(at));
        return table[at];
    };
    auto fetch = [&](int t, int entry, Codes &z) __attribute__((always_inline)) {
        const int page = t + 16 * (wave & 3) < t1 ? __builtin_amdgcn_readfirstlane(entry) : 0;
        z.in = page >= 0 && page < a.c.pages;                            // uniform
        const int64_t run = a.c.run(z.in ? page : 0, h) + ((t + 16 * (wave & 3)) & pmask);
        const uint8_t *p = codes + run * (D / 2) + code_at, *q = scales + run * (D / 16) + scale_at;
        if (keys) {
            if constexpr (D == 128) {
                const uint4 x = *reinterpret_cast<const uint4 *>(p);
                z.w[0] = x.x; z.w[1] = x.y; z.w[2] = x.z; z.w[3] = x.w;
                z.s = *reinterpret_cast<const uint16_t *>(q);
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(p);
                z.w[0] = x.x; z.w[1] = x.y;
                z.s = *q;
            }
        } else if (has) {
            const uint4 x = *reinterpret_cast<const uint4 *>(p);
            z.w[0] = x.x; z.w[1] = x.y; z.w[2] = x.z; z.w[3] = x.w;
            z.s = *reinterpret_cast<const uint32_t *>(q);
        }
    };
    auto unpack = [&](int t, Codes &z, uint8_t *stage) __attribute__((always_inline)) {
        uint8_t *d = stage + put_at;
        if (!z.in) z.s = keys ? 0x7F7Fu : 0u;
        if (keys) {
            const h2 sc = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(z.s, kScaleUp, false);
            const h2 sc0 = {sc[0], sc[0]}, sc1 = {sc[1], sc[1]};
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                const h2 sj = j < 2 ? sc0 : sc1;
                const uint32_t x = __builtin_amdgcn_perm(z.w[j], z.w[j], 0x01010000u);
                const uint32_t y = __builtin_amdgcn_perm(z.w[j], z.w[j], 0x03030202u);
                *reinterpret_cast<uint4 *>(d + (j >> 1) * 1024 + (j & 1) * 512) =
                    make_uint4(scaled((x << 4) & kCodeMask, sj), scaled(x & kCodeMask, sj), scaled((y << 4) & kCodeMask, sj),
                               scaled(y & kCodeMask, sj));
            }
        } else if (has) {
            if (t + 64 > see_least) {
                // hidden values, as in the kernel above
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = t + 16 * (wave & 3) + my_tok + i;
                    const bool nan = ((z.s >> (8 * i)) & 0x7Fu) == 0x7Fu;
                    if (at >= t1 || nan) z.s &= ~(0xFFu << (8 * i));
                    if (at < t1 && nan) atomicMin(&bad[my_at >> 1], at);
                }
            }
            const h2 s0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(z.s, kScaleUp, false);
            const h2 s1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(z.s, kScaleUp, true);
            uint32_t x[8], y[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t lo = __builtin_amdgcn_perm(z.w[1], z.w[0], 0x04040000u + 0x01010101u * j);
                const uint32_t hi = __builtin_amdgcn_perm(z.w[3], z.w[2], 0x04040000u + 0x01010101u * j);
                x[2 * j] = scaled((lo << 4) & kCodeMask, s0);
                y[2 * j] = scaled((hi << 4) & kCodeMask, s1);
                x[2 * j + 1] = scaled(lo & kCodeMask, s0);
                y[2 * j + 1] = scaled(hi & kCodeMask, s1);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const auto px = D == 128 ? __builtin_amdgcn_permlane32_swap(x[j], x[j + 4], false, false)
                                         : __builtin_amdgcn_permlane16_swap(x[j], x[j + 4], false, false);
                const auto py = D == 128 ? __builtin_amdgcn_permlane32_swap(y[j], y[j + 4], false, false)
                                         : __builtin_amdgcn_permlane16_swap(y[j], y[j + 4], false, false);
                *reinterpret_cast<uint4 *>(d + (j / CPT) * 2048 + WD * (j % CPT) * 16) = make_uint4(px[0], py[0], px[1], py[1]);
            }
        }
    };

    // the first codes are on their way while the queries are made ready
    Codes z, z1;
    int entries[4] = {0, 0, 0, 0};
    if (t0 < t1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) entries[k] = page_of(t0 + 64 * k);
        fetch(t0, entries[0], z);
        fetch(t0 + 64, entries[1], z1);
    }
    h8 qf[C::F];
    float c, sum = 0.0f;
    Reference ref;
    {
        const uint16_t *src = a.q + (sq.q0 + qi) * a.ldq + (int64_t)hq * D + 8 * up;
        uint4 w[C::F];
#pragma unroll
        for (int j = 0; j < C::F; ++j) w[j] = *reinterpret_cast<const uint4 *>(src + 16 * j);
        uint32_t top = largest(w);
        const uint32_t x = __shfl_xor(top, 32, 64);
        const int shift = row_shift(top > x ? top : x);
#pragma unroll
        for (int j = 0; j < C::F; ++j) qf[j] = query_f16(w[j], shift);
        c = score_factor(a, shift);
        ref.none(c);
    }
    // Operand m of a block: the products with 32 tokens' values (sub) and with the keys of 32 later ones, in turn.
    auto operand = [&](const uint8_t *sub, const uint8_t *keys_at, int m) __attribute__((always_inline)) {
        const int i = m >> 1;
        return m & 1 ? *reinterpret_cast<const h8 *>(keys_at + i * 1024 + turned[i / (C::F / 4)])
                     : *reinterpret_cast<const h8 *>(sub + (C::F + 2 * (i % VT) + i / VT) * 1024 + lane * 16);
    };
    h8 ops[4];                                                           // the next four
    // A block: O += V^T P^T of the 32 tokens whose weights are p, the scores `ahead` of 32 later tokens, and the weights of
    // the 32 between (scores s, first token t), which replace p.  An MFMA takes 32 cycles and its wave issues the
    // exponential of one element and the operand read four MFMAs ahead beside it: pinned in this order, since a wave
    // issues in order and stands still where two MFMAs meet.  The reference needs no maximum as long as
    // the sum of a lane's weights stays below the largest single one allowed.
    auto block = [&](const uint8_t *sub, const uint8_t *keys_at, const uint8_t *sub2, const uint8_t *keys2, int t,
                     f32x16 &s, f32x16 &ahead, uint32_t (&p)[8], auto edge) __attribute__((always_inline)) {
        if constexpr (decltype(edge)::value) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (t + 8 * (v >> 2) + 4 * up + (v & 3) >= see) s[v] = -__builtin_inff();
        }
        constexpr int kOps = 2 * C::F, kEach = 16 / kOps;
        auto pack = [](float a, float b) {
            const h2 z = {(_Float16)a, (_Float16)b};
            return __builtin_bit_cast(uint32_t, z);
        };
        uint32_t w[8];
        float total = 0.0f, e[2], arg = __builtin_fmaf(s[0], c, -ref.r);
#pragma unroll
        for (int v = 0; v < 16; ++v) ahead[v] = 0.0f;
        __builtin_amdgcn_sched_barrier(0);
        static_for<0, kOps>([&](auto M) __attribute__((always_inline)) {
            constexpr int m = M, i = m >> 1, x = i % VT, kc = i / VT;
            if constexpr (m & 1) ahead = __builtin_amdgcn_mfma_f32_32x32x16_f16(ops[m & 3], qf[i], ahead, 0, 0, 0);
            else o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ops[m & 3], frag(p[4 * kc], p[4 * kc + 1], p[4 * kc + 2], p[4 * kc + 3]), o[x], 0, 0, 0);
            if constexpr (m + 4 < kOps) ops[m & 3] = operand(sub, keys_at, m + 4);
            else ops[m & 3] = operand(sub2, keys2, m + 4 - kOps);
#pragma unroll
            for (int y = 0; y < kEach; ++y) {
                const int v = m * kEach + y;
                const float now = __builtin_amdgcn_exp2f(arg);           // used one element later: it takes a while
                if (v < 15) arg = __builtin_fmaf(s[(v + 1) & 15], c, -ref.r);
                if (v > 0) total += e[(v - 1) & 1];
                if (v > 0 && !(v & 1)) w[(v - 2) >> 1] = pack(e[0], e[1]);
                e[v & 1] = now;
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        total += e[1];
        w[7] = pack(e[0], e[1]);
        if (__any(!(total <= kMostSum))) {                               // or NaN, as in the kernel above
            float top = s[0];
#pragma unroll
            for (int v = 1; v < 16; ++v) top = __builtin_fmaxf(top, s[v]);
            top = __builtin_fmaxf(top, __shfl_xor(top, 32, 64));
            float f = 1.0f;
            if (ref.outgrown(top, c, __builtin_fmaxf(total, __shfl_xor(total, 32, 64)))) f = ref.renew(top, c);   // by the row's own scores alone
            sum *= f;
#pragma unroll
            for (int x = 0; x < VT; ++x)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[x][v] *= f;
            total = 0.0f;
#pragma unroll
            for (int v = 0; v < 16; v += 2) {
                const float e0 = ref.weight(s[v], c), e1 = ref.weight(s[v + 1], c);
                total += e0;
                total += e1;
                w[v >> 1] = pack(e0, e1);
            }
        }
        sum += total;
#pragma unroll
        for (int v = 0; v < 8; ++v) p[v] = w[v];
    };

    __syncthreads();                                                     // bad[] is set
    if (t0 < t1) {
        // Slots of the ring: the step before (its last values are still to come), this one, the next, and the one unpacked
        // into.  The last steps unpack what lies beyond the tokens (of page 0), which nothing uses.
        uint32_t slot = 0;
        auto stage = [&](uint32_t k) { return ring + (k & 3) * C::kStage; };
        unpack(t0, z, stage(0));
        unpack(t0 + 64, z1, stage(1));
        fetch(t0 + 128, entries[2], z);
        int page = entries[3], t = t0;
        __syncthreads();
        f32x16 s0, s1;
#pragma unroll
        for (int v = 0; v < 16; ++v) s0[v] = 0.0f;
#pragma unroll
        for (int i = 0; i < C::F; ++i) s0 = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand(ring, ring, 2 * i + 1), qf[i], s0, 0, 0, 0);
        uint32_t p[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const uint8_t *before = ring + C::kSub;                          // no weights yet
#pragma unroll
        for (int m = 0; m < 4; ++m) ops[m] = operand(before, ring + C::kSub, m);
        auto turn = [&]() __attribute__((always_inline)) {
            unpack(t + 128, z, stage(slot + 2));
            fetch(t + 192, page, z);
            page = page_of(t + 256);
        };
        // the waves of a SIMD (one with keys, one with values) unpack in different halves of a step; a wave without rows
        // does nothing else
        const bool busy = row0 + 32 * wave < rows;                       // uniform
        auto step = [&](auto edge) __attribute__((always_inline)) {
            const uint8_t *now = stage(slot), *next = stage(slot + 1);
            if (keys) turn();
            __builtin_amdgcn_s_setprio(1);                               // matrix instructions before the other wave's unpacking
            if (busy) block(before, now + C::kSub, now, next, t, s0, s1, p, edge);
            __builtin_amdgcn_s_setprio(0);
            if (!keys) turn();
            __builtin_amdgcn_s_setprio(1);
            if (busy) block(now, next, now + C::kSub, next + C::kSub, t + 32, s1, s0, p, edge);
            __builtin_amdgcn_s_setprio(0);
            before = now + C::kSub;
            ++slot;
            t += 64;
            __syncthreads();
        };
        const int open = t1 < wsee_least ? t1 : wsee_least;              // steps below it hide nothing from this wave
        while (t + 64 <= open) step(std::false_type{});
        while (t < t1) step(std::true_type{});
#pragma unroll
        for (int i = 0; i < C::F; ++i) {
            const int x = i % VT, kc = i / VT;
            o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand(before, before, 2 * i),
                                                          frag(p[4 * kc], p[4 * kc + 1], p[4 * kc + 2], p[4 * kc + 3]), o[x], 0, 0, 0);
        }
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < VT; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int w = (8 * (v >> 2) + 4 * up + (v & 3)) % WD;
            if (bad[w >> 1] < see) o[x][v] = __builtin_nanf("");
        }

    // rows through LDS, each wave in its own part, then out eight channels a lane
    constexpr int kLd = D + 1, kPer = D / 8;                             // lanes of a row
    float *mine = reinterpret_cast<float *>(ring) + wave * 32 * kLd;
    float *po = reinterpret_cast<float *>(a.workspace);
    const int64_t all = a.B * a.max_q * a.q_heads, at = (b * a.max_q + qi) * a.q_heads + hq;   // as in the kernel above
    sum += __shfl_xor(sum, 32, 64);
    const bool none = see == 0 && !sq.lost;
    const float f = splits > 1 ? 1.0f : finish_factor(sq.lost, none, sum), g1 = splits > 1 ? 1.0f : *a.c.gv;
    if (up == 0 && there) {
        if (splits > 1) {
            reinterpret_cast<PieceRow *>(po + (int64_t)splits * all * D)[split * all + at] = {ref.at(c), sum, 0.0f};
        } else if (a.lse) {
            a.lse[(sq.q0 + qi) * a.q_heads + hq] = sq.lost ? __builtin_nanf("") : none ? -__builtin_inff() : log_sum(ref.at(c), sum);
        }
    }
#pragma unroll
    for (int x = 0; x < VT; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int rho = 8 * (v >> 2) + 4 * up + (v & 3);
            mine[col * kLd + 8 * (rho % WD) + CPT * x + rho / WD] = none ? 0.0f : o[x][v] * f * g1;
        }
    __builtin_amdgcn_wave_barrier();
    const int64_t my_out = splits > 1 ? (split * all + at) * D : (sq.q0 + qi) * a.ldo + (int64_t)hq * D;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += 64 / kPer) {
        const int rr = r0 + lane / kPer, ch = lane % kPer * 8;
        const int64_t out = ((int64_t)__shfl((int)(my_out >> 32), rr, 64) << 32) | (uint32_t)__shfl((int)my_out, rr, 64);
        if (row0 + 32 * wave + rr < rows) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = mine[rr * kLd + ch + e];
            if (splits > 1) {
                float4 *dst = reinterpret_cast<float4 *>(po + out + ch);
                dst[0] = make_float4(y[0], y[1], y[2], y[3]);
                dst[1] = make_float4(y[4], y[5], y[6], y[7]);
            } else {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = bf16_rne_from_float(y[2 * e]) | (bf16_rne_from_float(y[2 * e + 1]) << 16);
                *reinterpret_cast<uint4 *>(a.out + out + ch) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

// Joins the splits of a row: one workgroup of W waves per query and head, a wave up to S of the splits.  Every load
// is on its way before the first is waited for; what was not written is not used.  A few rows: bound by the launch and
// one trip to memory (4.1 us for 40 rows of 64 splits); many: 18 MB in 6.4 us (2560 rows of up to 11).
template <int D, int W, int S>
__global__ __launch_bounds__(64 * W) void kv4_join_kernel(const Kv4AttnArgs a, int splits, int chunk) {
    constexpr int C = D / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hq = blockIdx.x % a.q_heads;
    const int64_t bi = blockIdx.x / a.q_heads;
    const int i = (int)(bi % a.max_q), b = (int)(bi / a.max_q);
    const Seq sq = sequence(a, b);
    if (i >= sq.nq) return;
    const int64_t all = a.B * a.max_q * a.q_heads;
    const float *po = reinterpret_cast<const float *>(a.workspace);
    const PieceRow *pm = reinterpret_cast<const PieceRow *>(po + (int64_t)splits * all * D);
    double ref[S];
    float weight[S], y[S][C];
#pragma unroll
    for (int k = 0; k < S; ++k) {
        const int s = wave + k * W;
        const int64_t slot = (s < splits ? s : 0) * all + bi * a.q_heads + hq;
        ref[k] = pm[slot].at;
        weight[k] = pm[slot].sum;
#pragma unroll
        for (int e = 0; e < C; ++e) y[k][e] = po[slot * D + lane * C + e];
    }
    const int n = visible(a, sq, i);
    const int have = sq.lost ? 0 : (n + chunk - 1) / chunk;              // the splits with a token that the row sees
    double m = kNoPiece;
#pragma unroll
    for (int k = 0; k < S; ++k)
        if (wave + k * W < have) m = __builtin_fmax(m, ref[k]);
    float total = 0.0f, z[C] = {};
#pragma unroll
    for (int k = 0; k < S; ++k)
        if (wave + k * W < have) {
            const float f = exp2_of(ref[k] - m);
            total = __builtin_fmaf(weight[k], f, total);
#pragma unroll
            for (int e = 0; e < C; ++e) z[e] = __builtin_fmaf(y[k][e], f, z[e]);
        }
    if constexpr (W > 1) {
        __shared__ float part[W][C + 1][64];
        __shared__ double tops[W];
#pragma unroll
        for (int e = 0; e < C; ++e) part[wave][e][lane] = z[e];
        part[wave][C][lane] = total;
        if (lane == 0) tops[wave] = m;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 1; w < W; ++w) m = __builtin_fmax(m, tops[w]);
        total = 0.0f;
#pragma unroll
        for (int e = 0; e < C; ++e) z[e] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = exp2_of(tops[w] - m);
            total = __builtin_fmaf(part[w][C][lane], f, total);
#pragma unroll
            for (int e = 0; e < C; ++e) z[e] = __builtin_fmaf(part[w][e][lane], f, z[e]);
        }
    }
    const bool none = n == 0 && !sq.lost;
    const float f = finish_factor(sq.lost, none, total), g1 = *a.c.gv;
    uint16_t *dst = a.out + (sq.q0 + i) * a.ldo + (int64_t)hq * D + lane * C;
    if constexpr (C == 2) *reinterpret_cast<uint32_t *>(dst) = bf16_rne_from_float(z[0] * f * g1) | (bf16_rne_from_float(z[1] * f * g1) << 16);
    else dst[0] = (uint16_t)bf16_rne_from_float(z[0] * f * g1);
    if (a.lse && lane == 0)
        a.lse[(sq.q0 + i) * a.q_heads + hq] = sq.lost ? __builtin_nanf("") : none ? -__builtin_inff() : log_sum(m, total);
}

template <int D, int NT, int W> void decode(const Kv4AttnArgs &a, const Kv4Plan &p, hipStream_t stream) {
    const int64_t n = a.B * a.c.heads * p.splits;
    kv4_decode_kernel<D, NT, W><<<(unsigned)n, 64 * W, 0, stream>>>(a, p.splits, p.chunk);
}

template <int D> void join(const Kv4AttnArgs &a, const Kv4Plan &p, hipStream_t stream) {
    const unsigned n = (unsigned)(a.B * a.max_q * a.q_heads);
    if (p.splits <= 4) kv4_join_kernel<D, 1, 4><<<n, 64, 0, stream>>>(a, p.splits, p.chunk);
    else if (p.splits <= 16) kv4_join_kernel<D, 4, 4><<<n, 256, 0, stream>>>(a, p.splits, p.chunk);
    else if (p.splits <= 32) kv4_join_kernel<D, 8, 4><<<n, 512, 0, stream>>>(a, p.splits, p.chunk);
    else if (p.splits <= 64) kv4_join_kernel<D, 8, 8><<<n, 512, 0, stream>>>(a, p.splits, p.chunk);
    else if (p.splits <= 128) kv4_join_kernel<D, 8, 16><<<n, 512, 0, stream>>>(a, p.splits, p.chunk);
    else kv4_join_kernel<D, 16, 16><<<n, 1024, 0, stream>>>(a, p.splits, p.chunk);
}

template <int D> hipError_t attend(const Kv4AttnArgs &a, const Kv4Plan &p, hipStream_t stream) {
    if (p.tiles == 1 && p.waves == 8) {
        decode<D, 1, 8>(a, p, stream);
    } else if (p.tiles == 1) {
        decode<D, 1, 4>(a, p, stream);
    } else if (p.tiles == 2) {
        decode<D, 2, 4>(a, p, stream);
    } else {
        const int64_t n = a.B * a.c.heads * p.splits * p.qtiles;
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kv4_prompt_kernel<D>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, Prompt<D>::kLds);
        if (e != hipSuccess) return e;
        kv4_prompt_kernel<D><<<(unsigned)n, 512, Prompt<D>::kLds, stream>>>(a, (int)p.qtiles, p.splits, p.chunk);
    }
    if (p.splits > 1) join<D>(a, p, stream);
    return hipGetLastError();
}

}  // namespace

size_t kv4_attention_workspace_bytes(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads, int D) {
    return (size_t)kv4_piece_rows(B, max_q, max_kv, q_heads, kv_heads) * ((size_t)D * 4 + sizeof(PieceRow));
}

hipError_t launch_kv4_attention(const Kv4AttnArgs &a, hipStream_t stream) {
    const Kv4Plan p = kv4_plan(a.B, a.max_q, a.max_kv, a.q_heads, a.c.heads);
    return a.c.D == 128 ? attend<128>(a, p, stream) : attend<64>(a, p, stream);
}

}  // namespace reqat
