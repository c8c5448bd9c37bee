// Internal launcher interface between the C ABI layer and the kernels.
// Every launcher only enqueues work on `stream` and returns hipGetLastError().
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dispatch.h"
#include "kv4_cache.h"
#include "kv4_plan.h"
#include "norm_plan.h"
#include "policy_plan.h"

namespace reqat {

// Maximum number of partial maxima the absmax pass produces; the workspace
// holds one uint32 per partial.
#ifndef REQAT_MAX_PARTIALS
#define REQAT_MAX_PARTIALS 4096
#endif
constexpr int kMaxPartials = REQAT_MAX_PARTIALS;

// Segment-table capacity of the quantize workspace (segments of 64 blocks).
constexpr int64_t kMaxSegments = int64_t(1) << 19;

// Output selector for the block quantizer.
// kBoth writes codes, scales and fake-quant values in one pass over x.
enum QuantOut : int { kCodes = 0, kFakeQuant = 1, kBoth = 2 };

// Global-scale source for NVFP4.
enum GSrc : int { kGComputed = 0, kGGiven = 1, kGNone = 2 };

hipError_t launch_unit_scale(float *gptr, hipStream_t stream);

hipError_t launch_absmax(const uint16_t *x, int64_t rows, int64_t cols, int64_t ldx,
                         uint32_t *partials, int *nparts_out, hipStream_t stream);

// NVFP4 with a computed g reads x once when the segment table (one uint16 per
// 64 blocks) has room for the tensor, and twice (absmax pass first) otherwise.
hipError_t launch_quantize(Fmt fmt, QuantOut out, const uint16_t *x, int64_t rows, int64_t cols,
                           int64_t ldx, uint8_t *codes, uint8_t *scales, uint16_t *y, int64_t ldy,
                           float *gptr, GSrc gsrc, uint32_t *partials, uint16_t *seg_table,
                           int64_t seg_capacity, hipStream_t stream);

// MXFP4 quantize / fake-quant of block-rotated rows (randomized Hadamard of 32).
hipError_t launch_quantize_rht(QuantOut out, const uint16_t *x, int64_t rows, int64_t cols, int64_t ldx,
                               uint32_t signs, uint8_t *codes, uint8_t *scales, uint16_t *y, int64_t ldy,
                               hipStream_t stream);

// W4A16: bfloat16 x [M][ldx] times MXFP4 weights [N][K/2] (+ scales [N][K/32]), K % 128 == 0.
// `workspace` holds gemm_w4a16_workspace_bytes(M, N, K) bytes of split-K partial sums.
size_t gemm_w4a16_workspace_bytes(int64_t M, int64_t N, int64_t K);
// Tiles (gemm_w4a16_tile.hip): 0 < K <= kW16TileMaxLd, K % 128 == 0, ldx <= kW16TileMaxLd; packed as below.
hipError_t launch_gemm_w4a16_tile(W16Tile tile, int64_t M, int64_t N, int64_t K, const uint16_t *x, int64_t ldx,
                                  const uint8_t *w_codes, const uint8_t *w_scales, bool packed, void *y, bool y_bf16,
                                  int64_t ldy, hipStream_t stream);
// packed: w_codes / w_scales are the code and scale parts of the packed image
// that launch_w4a16_pack writes (w4a16_packed_bytes(N, K) bytes).
hipError_t launch_gemm_w4a16(int64_t M, int64_t N, int64_t K, const uint16_t *x, int64_t ldx,
                             const uint8_t *w_codes, const uint8_t *w_scales, bool packed, void *y, bool y_bf16,
                             int64_t ldy, float *workspace, hipStream_t stream);
size_t w4a16_packed_bytes(int64_t N, int64_t K);
hipError_t launch_w4a16_pack(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t K, uint8_t *packed,
                             hipStream_t stream);

// KV4 (E1M2 elements, E4M3 block scales of 16, FP32 global scale) of x - shift.
// A computed g takes one pass over x and a fix-up kernel when the segment
// table (one uint16 per 64 blocks) has room for the tensor, else an absmax pass
// into `partials` (<= kMaxPartials) and then the quantizer.
hipError_t launch_kv4(QuantOut out, const uint16_t *x, int64_t rows, int64_t cols, int64_t ldx, const float *shift,
                      uint8_t *codes, uint8_t *scales, uint16_t *y, int64_t ldy, float *gptr, bool computed,
                      uint32_t *partials, uint16_t *seg_table, hipStream_t stream);

// Paged KV4 cache (kv4_cache.hip): D is 64 or 128.  q may be null (q_heads 0); cos null: no rotation.
hipError_t launch_kv4_append(const Kv4View &c, int64_t T, const int64_t *slots, const uint16_t *k, int64_t ldk,
                             const uint16_t *v, int64_t ldv, const uint16_t *q, int64_t ldq, int q_heads,
                             uint16_t *q_out, int64_t ldq_out, const float *cos, const float *sin,
                             const int32_t *positions, int64_t rope_len, hipStream_t stream);
// k or v may be null.
hipError_t launch_kv4_gather(const Kv4View &c, int64_t T, const int64_t *slots, uint16_t *k, int64_t ldk, uint16_t *v,
                             int64_t ldv, bool add_shift, hipStream_t stream);

// Attention over the cache (kv4_attention.hip).
struct Kv4AttnArgs {
    Kv4View c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;                            // [T][q_heads] or null
    const int32_t *q_start, *kv_len, *table;
    int64_t B, T, ldq, ldo, ld_table, table_cols, max_q, max_kv;
    int q_heads;
    bool causal;
    float scale;
    void *workspace;
};
size_t kv4_attention_workspace_bytes(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads, int D);
hipError_t launch_kv4_attention(const Kv4AttnArgs &a, hipStream_t stream);

// SEM loss: per-row statistics ([T][4]: H, NLL, lse, 0), weights [T], loss[4]
// (L, L_SFT, L_ent, tau); backward writes dL/dlogits.  V % 8 == 0.
hipError_t launch_sem_forward(const uint16_t *logits, int64_t T, int64_t V, int64_t ld, const int32_t *targets,
                              float lambda, float eps, float *stats, float *weights, float *loss,
                              hipStream_t stream);
hipError_t launch_sem_backward(const uint16_t *logits, int64_t T, int64_t V, int64_t ld, const int32_t *targets,
                               const float *stats, const float *weights, float lambda, float scale, void *grad,
                               bool grad_bf16, int64_t ldg, hipStream_t stream);

// Policy loss (policy.hip).  stats [T][4]: lp, log-sum-exp, dL/dlp, ratio; loss [4].
struct PolicyArgs {
    const void *logits;                    // [T][ld] bfloat16 or FP32
    const int32_t *targets;
    const float *old_logp, *adv, *ref;     // ref null: no KL term
    const float *weights;                  // null: default_weight for every token
    float *stats, *loss;
    void *grad;                            // [T][ldg] of the logits' type, or null
    const float *grad_loss;                // backward: dL's factor on the device, or null
    float4 *parts;                         // workspace: the statistics of policy_plan's slices
    int64_t T, V, ld, ldg;
    float default_weight, low, high;       // low, high: bounds of the ratio
    float kl, temp;
    float c, c_rest;                       // log2(e) / temperature: rounded; FP32: rounded down, and what that leaves, > 0
};
// The statistics and the loss, and the gradient where a.grad is not null.
hipError_t launch_policy_loss(const PolicyArgs &a, bool bf16, hipStream_t stream);
// The gradient from logits, targets and stats.
hipError_t launch_policy_backward(const PolicyArgs &a, bool bf16, hipStream_t stream);

// Layer norm (norm.hip), K <= kNormMaxCols.  stats [M][2]: mean, 1 / standard deviation.
struct NormArgs {
    const void *x, *dy, *w, *b;            // x, dy, y, dx of one type; w, b, dw, db of another; b, db may be null
    void *y, *dx, *dw, *db;
    float *stats, *partials;               // partials: norm_plan's sums x K of dw, then of db
    int64_t M, K, ldx, lddy, ldy, lddx;
    float eps;
    bool center, w_bf16;
};
hipError_t launch_norm(const NormArgs &a, bool bf16, bool backward, hipStream_t stream);

// Embedding (embedding.hip).
constexpr int kEmbedPiece = 16;            // sorted tokens whose rows one wave adds up
struct EmbedArgs {
    const int32_t *ids;
    const void *table;
    void *out;
    int64_t T, V, D, ld_table, ld_out;
    float scale;
};
hipError_t launch_embedding(const EmbedArgs &a, bool bf16, hipStream_t stream);
struct EmbedGradArgs {
    const void *dy;
    void *dtable;
    int32_t *valid;                        // workspace (null where none is needed)
    int4 *places;
    float *partials;
    int64_t T, V, D, ld_dy, ld_table;
    float scale;
    bool accumulate;
};
size_t embedding_workspace_bytes(int64_t T, int64_t V, int64_t D);
hipError_t launch_embedding_backward(const EmbedGradArgs &a, const int32_t *ids, bool bf16, bool table_bf16, hipStream_t stream);

// AdamW (adamw.hip).
constexpr int kAdamBlock = 128;            // elements to a scale of the 8-bit states
struct AdamTensor {
    void *p;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale;
    void *copy;
    int64_t n;
};
struct AdamCoef {
    float b1, c1, b2, c2, decay, step, root, eps;
};
hipError_t launch_adamw(const AdamTensor *tensors, int64_t count, bool p_bf16, bool g_bf16, int bits, const AdamCoef &c,
                        const float *dev_coef, const float *grad_scale, hipStream_t stream);
hipError_t launch_adamw_coef(double lr, double beta1, double beta2, double decay, const float *lr_dev, int32_t *step,
                             float *coef, hipStream_t stream);
hipError_t launch_adamw_moments(const uint8_t *mc, const float *ms, const uint8_t *vc, const float *vs, int64_t n, float *m,
                                float *v, hipStream_t stream);

bool gemm_tile256_supported(Fmt fmt, int64_t M, int64_t N, int64_t K, int64_t ldy);
// Skinny product for M <= 64 (K % 128 == 0, K > 0).  packed: b_codes / b_scales
// are the code and scale parts of the image launch_skinny_pack writes
// (skinny_packed_bytes(fmt, N, K) bytes; the scales start 2048 G C bytes in).
hipError_t launch_gemm_skinny(Fmt fmt, int64_t M, int64_t N, int64_t K, const uint8_t *a_codes,
                              const uint8_t *a_scales, const float *ga, const uint8_t *b_codes,
                              const uint8_t *b_scales, const float *gb, void *y, bool y_bf16, int64_t ldy,
                              bool packed, hipStream_t stream);
size_t skinny_packed_bytes(Fmt fmt, int64_t N, int64_t K);
hipError_t launch_skinny_pack(Fmt fmt, const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t K,
                              uint8_t *packed, hipStream_t stream);

hipError_t launch_gemm_tile256(Fmt fmt, int64_t M, int64_t N, int64_t K, const uint8_t *a_codes,
                               const uint8_t *a_scales, const float *ga, const uint8_t *b_codes,
                               const uint8_t *b_scales, const float *gb, void *y, bool y_bf16,
                               int64_t ldy, hipStream_t stream);

// Small tiles (gemm_ksplit.hip): 0 < K <= kKsplitMaxK, K % 128 == 0.
hipError_t launch_gemm_ksplit(KsplitTile tile, Fmt fmt, int64_t M, int64_t N, int64_t K, const uint8_t *a_codes,
                              const uint8_t *a_scales, const float *ga, const uint8_t *b_codes,
                              const uint8_t *b_scales, const float *gb, void *y, bool y_bf16, int64_t ldy,
                              bool packed, hipStream_t stream);

// M <= 64 and K > 0; packed: b_codes / b_scales are the parts of the decode image.
hipError_t launch_gemm_decode(Fmt fmt, int64_t M, int64_t N, int64_t K, const uint8_t *a_codes,
                              const uint8_t *a_scales, const float *ga, const uint8_t *b_codes,
                              const uint8_t *b_scales, const float *gb, void *y, bool y_bf16, int64_t ldy,
                              bool packed, hipStream_t stream);

hipError_t launch_gemm(Fmt fmt, int64_t M, int64_t N, int64_t K, const uint8_t *a_codes,
                       const uint8_t *a_scales, const float *ga, const uint8_t *b_codes,
                       const uint8_t *b_scales, const float *gb, void *y, bool y_bf16, int64_t ldy,
                       hipStream_t stream);

}  // namespace reqat
