// C ABI of libreqat, training side: the operators around the quantized linear layers (embedding, norm, policy loss, AdamW).
// Argument validation as in api.hip: on the host, before any HIP call.
#include <math.h>

#include "../../include/reqat.h"
#include "internal.h"
#include "row_overlap.h"

namespace {

using namespace reqat;

constexpr int64_t kMaxTokens = 1 << 22;               // a launch's threads stay below 2^32
constexpr int64_t kMaxVocab = 1 << 23;

bool dtype_ok(reqat_dtype d) { return d == REQAT_DT_F32 || d == REQAT_DT_BF16; }
int64_t size_of(reqat_dtype d) { return d == REQAT_DT_BF16 ? 2 : 4; }

// Aligned to n bytes, a power of two.
bool aligned(const void *p, int64_t n) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(n - 1)) == 0; }

// A matrix as the overlap test takes it, in units of two bytes.
struct Rows {
    const void *p;
    int64_t rows, cols, ld, size;
};
bool overlap(const Rows &a, const Rows &b) {
    if (a.rows == 0 || b.rows == 0) return false;     // the strides of no rows may be anything
    return rows_overlap(a.p, a.rows, a.cols * a.size / 2, a.ld * a.size / 2, b.p, b.rows, b.cols * b.size / 2, b.ld * b.size / 2);
}
bool in_place(const Rows &a, const Rows &b) { return a.p == b.p && (a.ld == b.ld || a.rows == 1) && a.size == b.size; }

// The last element's offset fits 62 bits, in bytes too.
bool span_ok(int64_t rows, int64_t ld) { return ld >= 0 && (rows <= 0 || ld <= (int64_t(1) << 59) / rows); }

}  // namespace

extern "C" {

static reqat_status check_policy(const void *logits, reqat_dtype dtype, int64_t T, int64_t V, int64_t ld, const int32_t *targets,
                                 float temperature, const float *stats, const void *grad, int64_t ldg, bool need_grad) {
    if (!dtype_ok(dtype)) return REQAT_E_ENUM;
    if (T < 0 || T > kMaxTokens || V <= 0 || V > (1 << 30) || ld < V || !span_ok(T, ld)) return REQAT_E_SHAPE;
    if (need_grad && (ldg < V || !span_ok(T, ldg))) return REQAT_E_SHAPE;
    if (!(temperature >= 1.17549435e-38f) || isinf(temperature)) return REQAT_E_UNSUPPORTED;   // 2^-126: log2(e) / temperature is finite
    if (T == 0) return REQAT_OK;
    if (!logits || !targets || !stats || (need_grad && !grad)) return REQAT_E_NULL;
    if (!aligned(logits, size_of(dtype)) || !aligned(targets, 4) || !aligned(stats, 16) || !aligned(grad, size_of(dtype)))
        return REQAT_E_ALIGN;
    if (need_grad) {
        const Rows z{logits, T, V, ld, size_of(dtype)}, g{grad, T, V, ldg, size_of(dtype)};
        if (!in_place(z, g) && overlap(z, g)) return REQAT_E_UNSUPPORTED;
    }
    return REQAT_OK;
}

static void set_temperature(PolicyArgs &a, float temperature, bool bf16) {
    const double c = 1.4426950408889634074 / (double)temperature;
    a.temp = temperature;
    a.c = (float)c;
    if (bf16) return;
    if ((double)a.c >= c) a.c = nextafterf(a.c, 0.0f);
    const float rest = (float)(c - (double)a.c);
    a.c_rest = rest > 0.0f ? rest : 1e-45f;              // never 0, which -Inf times would be NaN
}

size_t reqat_policy_loss_workspace_bytes(reqat_dtype dtype, int64_t T, int64_t V) {
    if (!dtype_ok(dtype) || T < 0 || T > kMaxTokens || V <= 0 || V > (1 << 30)) return 0;
    const PolicyPlan p = policy_plan(T, V, dtype == REQAT_DT_BF16);
    return p.slices > 1 ? (size_t)(T * p.slices) * 16 : 0;
}

reqat_status reqat_policy_loss(const void *logits, reqat_dtype dtype, int64_t T, int64_t V, int64_t ld, const int32_t *targets,
                               const float *old_logp, const float *advantages, const float *ref_logp, const float *weights,
                               float clip_low, float clip_high, float kl_coef, float temperature, float *stats, float *loss,
                               void *grad, int64_t ldg, void *workspace, void *stream) {
    const reqat_status st = check_policy(logits, dtype, T, V, ld, targets, temperature, stats, grad, ldg, grad != nullptr);
    if (st != REQAT_OK) return st;
    if (!workspace && reqat_policy_loss_workspace_bytes(dtype, T, V) > 0) return REQAT_E_NULL;
    if (!aligned(workspace, 16)) return REQAT_E_ALIGN;
    if (!(clip_low >= 0.0f) || !(clip_low <= 1.0f) || !(clip_high >= 0.0f)) return REQAT_E_UNSUPPORTED;
    if (!loss || (T > 0 && (!old_logp || !advantages || (kl_coef != 0.0f && !ref_logp)))) return REQAT_E_NULL;
    if (!aligned(loss, 4) || !aligned(old_logp, 4) || !aligned(advantages, 4) || !aligned(ref_logp, 4) || !aligned(weights, 4))
        return REQAT_E_ALIGN;
    PolicyArgs a = {};
    a.logits = logits; a.targets = targets; a.old_logp = old_logp; a.adv = advantages; a.weights = weights;
    a.ref = ref_logp; a.stats = stats; a.loss = loss; a.grad = grad; a.parts = reinterpret_cast<float4 *>(workspace);
    a.T = T; a.V = V; a.ld = ld; a.ldg = ldg;
    a.default_weight = T > 0 ? (float)(1.0 / (double)T) : 0.0f;
    a.low = (float)(1.0 - (double)clip_low);
    a.high = (float)(1.0 + (double)clip_high);
    a.kl = kl_coef;
    set_temperature(a, temperature, dtype == REQAT_DT_BF16);
    return launch_policy_loss(a, dtype == REQAT_DT_BF16, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

reqat_status reqat_policy_loss_backward(const void *logits, reqat_dtype dtype, int64_t T, int64_t V, int64_t ld,
                                        const int32_t *targets, const float *stats, float temperature, const float *grad_loss,
                                        void *grad, int64_t ldg, void *stream) {
    const reqat_status st = check_policy(logits, dtype, T, V, ld, targets, temperature, stats, grad, ldg, true);
    if (st != REQAT_OK) return st;
    if (!aligned(grad_loss, 4)) return REQAT_E_ALIGN;
    PolicyArgs a = {};
    a.logits = logits; a.targets = targets; a.stats = const_cast<float *>(stats); a.grad_loss = grad_loss; a.grad = grad;
    a.T = T; a.V = V; a.ld = ld; a.ldg = ldg;
    set_temperature(a, temperature, dtype == REQAT_DT_BF16);
    return launch_policy_backward(a, dtype == REQAT_DT_BF16, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

static reqat_status check_norm(reqat_dtype dtype, reqat_dtype w_dtype, int64_t rows, int64_t cols) {
    if (!dtype_ok(dtype) || !dtype_ok(w_dtype)) return REQAT_E_ENUM;
    if (rows < 0 || cols <= 0 || rows > (int64_t(1) << 40)) return REQAT_E_SHAPE;
    return cols > kNormMaxCols ? REQAT_E_UNSUPPORTED : REQAT_OK;
}

reqat_status reqat_layer_norm(const void *x, reqat_dtype dtype, int64_t rows, int64_t cols, int64_t ldx, const void *weight,
                              const void *bias, reqat_dtype w_dtype, float eps, int center, void *y, int64_t ldy, float *stats,
                              void *stream) {
    reqat_status st = check_norm(dtype, w_dtype, rows, cols);
    if (st != REQAT_OK) return st;
    if (ldx < cols || ldy < cols || !span_ok(rows, ldx) || !span_ok(rows, ldy)) return REQAT_E_SHAPE;
    if (!(eps >= 0.0f) || isinf(eps)) return REQAT_E_UNSUPPORTED;
    if (rows == 0) return REQAT_OK;
    if (!x || !weight || !y || !stats) return REQAT_E_NULL;
    const int64_t e = size_of(dtype), w = size_of(w_dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(weight, w) || !aligned(bias, w) || !aligned(stats, 4)) return REQAT_E_ALIGN;
    const Rows in{x, rows, cols, ldx, e}, out{y, rows, cols, ldy, e};
    if (!in_place(in, out) && overlap(in, out)) return REQAT_E_UNSUPPORTED;
    NormArgs a = {};
    a.x = x; a.w = weight; a.b = bias; a.y = y; a.stats = stats;
    a.M = rows; a.K = cols; a.ldx = ldx; a.ldy = ldy;
    a.eps = eps; a.center = center != 0; a.w_bf16 = w_dtype == REQAT_DT_BF16;
    return launch_norm(a, dtype == REQAT_DT_BF16, false, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

size_t reqat_layer_norm_workspace_bytes(reqat_dtype dtype, int64_t rows, int64_t cols, int bias) {
    if (check_norm(dtype, REQAT_DT_F32, rows, cols) != REQAT_OK) return 0;
    return (size_t)norm_plan(rows, cols, dtype == REQAT_DT_BF16).sums * (size_t)cols * (bias ? 8 : 4);
}

reqat_status reqat_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, reqat_dtype dtype, int64_t rows,
                                       int64_t cols, const void *weight, reqat_dtype w_dtype, const float *stats, int center,
                                       void *dx, int64_t lddx, void *dweight, void *dbias, void *workspace, void *stream) {
    reqat_status st = check_norm(dtype, w_dtype, rows, cols);
    if (st != REQAT_OK) return st;
    if (lddy < cols || ldx < cols || lddx < cols || !span_ok(rows, lddy) || !span_ok(rows, ldx) || !span_ok(rows, lddx))
        return REQAT_E_SHAPE;
    if (!dweight || (rows > 0 && (!dy || !x || !weight || !stats || !dx || !workspace))) return REQAT_E_NULL;
    const int64_t e = size_of(dtype), w = size_of(w_dtype);
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dx, e) || !aligned(weight, w) || !aligned(dweight, w) || !aligned(dbias, w) ||
        !aligned(stats, 4) || !aligned(workspace, 4))
        return REQAT_E_ALIGN;
    const Rows up{dy, rows, cols, lddy, e}, in{x, rows, cols, ldx, e}, out{dx, rows, cols, lddx, e};
    if ((!in_place(up, out) && overlap(up, out)) || (!in_place(in, out) && overlap(in, out))) return REQAT_E_UNSUPPORTED;
    NormArgs a = {};
    a.dy = dy; a.x = x; a.w = weight; a.stats = const_cast<float *>(stats); a.dx = dx; a.dw = dweight; a.db = dbias;
    a.partials = reinterpret_cast<float *>(workspace);
    a.M = rows; a.K = cols; a.lddy = lddy; a.ldx = ldx; a.lddx = lddx;
    a.center = center != 0; a.w_bf16 = w_dtype == REQAT_DT_BF16;
    return launch_norm(a, dtype == REQAT_DT_BF16, true, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

static reqat_status check_embedding(int64_t T, int64_t V, int64_t D) {
    return T < 0 || T > kMaxTokens || V < 0 || V > kMaxVocab || D <= 0 || D > (1 << 20) || T > (int64_t(1) << 37) / D ? REQAT_E_SHAPE : REQAT_OK;
}

reqat_status reqat_embedding(const int32_t *ids, int64_t T, const void *table, reqat_dtype dtype, int64_t V, int64_t D,
                             int64_t ld_table, float scale, void *out, int64_t ldo, void *stream) {
    if (!dtype_ok(dtype)) return REQAT_E_ENUM;
    if (check_embedding(T, V, D) != REQAT_OK || ld_table < D || ldo < D || !span_ok(V, ld_table) || !span_ok(T, ldo)) return REQAT_E_SHAPE;
    if (T == 0) return REQAT_OK;
    if (!ids || !out || (V > 0 && !table)) return REQAT_E_NULL;
    const int64_t e = size_of(dtype);
    if (!aligned(ids, 4) || !aligned(table, e) || !aligned(out, e)) return REQAT_E_ALIGN;
    if (overlap({table, V, D, ld_table, e}, {out, T, D, ldo, e})) return REQAT_E_UNSUPPORTED;
    const EmbedArgs a = {ids, table, out, T, V, D, ld_table, ldo, scale};
    return launch_embedding(a, dtype == REQAT_DT_BF16, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

size_t reqat_embedding_workspace_bytes(int64_t T, int64_t V, int64_t D) {
    return check_embedding(T, V, D) == REQAT_OK ? embedding_workspace_bytes(T, V, D) : 0;
}

reqat_status reqat_embedding_backward(const void *dy, reqat_dtype dtype, int64_t lddy, const int32_t *ids, int64_t T, int64_t V,
                                      int64_t D, float scale, void *dtable, reqat_dtype table_dtype, int64_t ld_table,
                                      int accumulate, void *workspace, void *stream) {
    if (!dtype_ok(dtype) || !dtype_ok(table_dtype)) return REQAT_E_ENUM;
    if (check_embedding(T, V, D) != REQAT_OK || lddy < D || ld_table < D || !span_ok(T, lddy) || !span_ok(V, ld_table)) return REQAT_E_SHAPE;
    if (V == 0 || (T == 0 && accumulate)) return REQAT_OK;
    if (!dtable || (T > 0 && (!dy || !ids)) || (!workspace && embedding_workspace_bytes(T, V, D) > 0)) return REQAT_E_NULL;
    const int64_t e = size_of(dtype), g = size_of(table_dtype);
    if (!aligned(dy, e) || !aligned(ids, 4) || !aligned(dtable, g) || !aligned(workspace, 16)) return REQAT_E_ALIGN;
    if (overlap({dy, T, D, lddy, e}, {dtable, V, D, ld_table, g})) return REQAT_E_UNSUPPORTED;
    EmbedGradArgs a = {};
    a.dy = dy; a.dtable = dtable;
    if (workspace) {
        a.valid = reinterpret_cast<int32_t *>(workspace);
        a.places = reinterpret_cast<int4 *>(reinterpret_cast<uint8_t *>(workspace) + 16);
        a.partials = reinterpret_cast<float *>(a.places + T);
    }
    a.T = T; a.V = V; a.D = D; a.ld_dy = lddy; a.ld_table = ld_table;
    a.scale = scale; a.accumulate = accumulate != 0;
    return launch_embedding_backward(a, ids, dtype == REQAT_DT_BF16, table_dtype == REQAT_DT_BF16,
                                     reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

static reqat_status check_hyper(const reqat_adamw_hyper *h) {
    if (!h) return REQAT_E_NULL;
    const bool ok = isfinite(h->lr) && h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0 && h->eps >= 0.0 &&
                    isfinite(h->eps) && isfinite(h->weight_decay);
    return ok ? REQAT_OK : REQAT_E_UNSUPPORTED;
}

reqat_status reqat_adamw_step(const reqat_adamw_tensor *tensors, int64_t count, reqat_dtype p_dtype, reqat_dtype g_dtype,
                              int state_bits, const reqat_adamw_hyper *hyper, const float *grad_scale, const float *coef,
                              void *stream) {
    if (!dtype_ok(p_dtype) || !dtype_ok(g_dtype)) return REQAT_E_ENUM;
    if (count < 0) return REQAT_E_SHAPE;
    if (state_bits != 8 && state_bits != 32) return REQAT_E_UNSUPPORTED;
    const reqat_status st = check_hyper(hyper);
    if (st != REQAT_OK) return st;
    if (!coef && hyper->step < 1) return REQAT_E_UNSUPPORTED;
    if (!aligned(grad_scale, 4) || !aligned(coef, 4)) return REQAT_E_ALIGN;
    if (count > 0 && !tensors) return REQAT_E_NULL;
    const int64_t state = state_bits == 32 ? 4 : 1;
    for (int64_t i = 0; i < count; ++i) {
        const reqat_adamw_tensor &t = tensors[i];
        if (t.n < 0 || t.n > (int64_t(1) << 34)) return REQAT_E_SHAPE;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || (state_bits == 8 && (!t.m_scale || !t.v_scale))) return REQAT_E_NULL;
        if (!aligned(t.p, size_of(p_dtype)) || !aligned(t.g, size_of(g_dtype)) || !aligned(t.m, state) || !aligned(t.v, state) ||
            !aligned(t.copy, 2) || (state_bits == 8 && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
            return REQAT_E_ALIGN;
    }
    static_assert(sizeof(reqat_adamw_tensor) == sizeof(AdamTensor), "one layout");
    AdamCoef c = {};
    c.b1 = (float)hyper->beta1;
    c.c1 = (float)(1.0 - hyper->beta1);
    c.b2 = (float)hyper->beta2;
    c.c2 = (float)(1.0 - hyper->beta2);
    c.eps = (float)hyper->eps;
    if (!coef) {
        const double t = (double)hyper->step;
        c.decay = (float)(1.0 - hyper->lr * hyper->weight_decay);
        c.step = (float)(hyper->lr / -expm1(t * log(hyper->beta1)));
        c.root = (float)(1.0 / sqrt(-expm1(t * log(hyper->beta2))));
    }
    return launch_adamw(reinterpret_cast<const AdamTensor *>(tensors), count, p_dtype == REQAT_DT_BF16, g_dtype == REQAT_DT_BF16,
                        state_bits, c, coef, grad_scale, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

reqat_status reqat_adamw_coefficients(const reqat_adamw_hyper *hyper, const float *lr, int32_t *step, float *coef, void *stream) {
    const reqat_status st = check_hyper(hyper);
    if (st != REQAT_OK) return st;
    if (!step || !coef) return REQAT_E_NULL;
    if (!aligned(lr, 4) || !aligned(step, 4) || !aligned(coef, 4)) return REQAT_E_ALIGN;
    return launch_adamw_coef(hyper->lr, hyper->beta1, hyper->beta2, hyper->weight_decay, lr, step, coef,
                             reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? REQAT_OK : REQAT_E_HIP;
}

reqat_status reqat_adamw_moments(const uint8_t *m, const float *m_scale, const uint8_t *v, const float *v_scale, int64_t n,
                                 float *m_out, float *v_out, void *stream) {
    if (n < 0 || n > (int64_t(1) << 33)) return REQAT_E_SHAPE;
    if (n == 0) return REQAT_OK;
    if (!m || !m_scale || !v || !v_scale || !m_out || !v_out) return REQAT_E_NULL;
    if (!aligned(m_scale, 4) || !aligned(v_scale, 4) || !aligned(m_out, 4) || !aligned(v_out, 4)) return REQAT_E_ALIGN;
    return launch_adamw_moments(m, m_scale, v, v_scale, n, m_out, v_out, reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? REQAT_OK : REQAT_E_HIP;
}

}  // extern "C"
