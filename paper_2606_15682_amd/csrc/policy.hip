// Clipped policy loss with a KL term for gfx950, per token t (a row of logits z, p = softmax(z / temperature)):
//   lp = log p_y,  r = exp(lp - old),  x = ref - lp,
//   loss_t = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(x) - x - 1),   L = sum_t w_t loss_t,
//   dL/dlp = w_t (-A r [inside] - kl (exp(x) - 1)),  inside: neither A > 0, r > 1 + high nor A < 0, r < 1 - low,
//   dL/dz_j = (dL/dlp) ([j = y] - p_j) / temperature.
//
// Softmax statistics in base-2 units: c = log2(e) / temperature, mb = c max z, t = c z - mb in one fused multiply-add,
// S = sum 2^t; then lp = ln 2 (t_y - log2 S) and p_j = 2^t_j / S.  The rounding of mb is in every t alike and leaves lp and
// p as they are.
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

constexpr int kThreads = 512;

// Running maximum and sum of a slice of a row; empty: m = -Inf, mb = 0, S = 0, and so for a slice of -Inf logits alone.
struct Online {
    float m, mb, S;
};

__device__ __forceinline__ void grow(Online &o, float mx, float c) {
    if (mx > o.m) {
        const float mxb = mx * c;
        if (o.S != 0.0f) o.S *= __builtin_amdgcn_exp2f(o.mb - mxb);
        o.m = mx;
        o.mb = mxb;
    }
}

// A NaN logit makes S NaN, and so does +Inf (Inf - Inf): the row's statistics are NaN then.
template <int N> __device__ __forceinline__ void add(Online &o, const float (&z)[N], float c) {
    float mx = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) mx = __builtin_fmaxf(mx, z[i]);
    grow(o, mx, c);
#pragma unroll
    for (int i = 0; i < N; ++i) o.S += __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], c, -o.mb));
}

__device__ __forceinline__ Online merge(Online a, Online b) {
    if (b.m > a.m) { const Online t = a; a = b; b = t; }
    if (b.S == 0.0f) return a;
    a.S += b.S * __builtin_amdgcn_exp2f(b.mb - a.mb);
    return a;
}

// exp(x) - x - 1 >= 0.  Near zero the difference of close numbers is summed as its series (to x^8 / 8!: 2e-8 of it at 1/2).
__device__ __forceinline__ float kl_term(float x) {
    if (__builtin_fabsf(x) < 0.5f) {
        float s = 1.0f / 40320.0f;
        s = __builtin_fmaf(s, x, 1.0f / 5040.0f);
        s = __builtin_fmaf(s, x, 1.0f / 720.0f);
        s = __builtin_fmaf(s, x, 1.0f / 120.0f);
        s = __builtin_fmaf(s, x, 1.0f / 24.0f);
        s = __builtin_fmaf(s, x, 1.0f / 6.0f);
        s = __builtin_fmaf(s, x, 0.5f);
        return s * x * x;
    }
    return expm1f(x) - x;
}

__device__ __forceinline__ bool outside(const PolicyArgs &a, float r, float adv) {
    return (adv > 0.0f && r > a.high) || (adv < 0.0f && r < a.low);
}

__device__ __forceinline__ float weight_of(const PolicyArgs &a, int64_t t) {
    return a.weights ? a.weights[t] : a.default_weight;
}

// lp, log-sum-exp, dL/dlp and r of a row with weight w != 0.
__device__ __forceinline__ float4 row_stats(const PolicyArgs &a, int64_t t, float w, Online o, float zy) {
    const float log2S = __builtin_amdgcn_logf(o.S);
    const float lp = (__builtin_fmaf(zy, a.c, -o.mb) - log2S) * kLn2;
    const float r = expf(lp - a.old_logp[t]), adv = a.adv[t];
    float slope = outside(a, r, adv) ? 0.0f : -adv * r;
    if (a.ref) slope -= a.kl * expm1f(a.ref[t] - lp);
    return make_float4(lp, (o.mb + log2S) * kLn2, w * slope, r);
}

// 0 <= y < V, else NaN without a read.
template <typename T> __device__ __forceinline__ float target_logit(const PolicyArgs &a, const T *row, int32_t y) {
    return y >= 0 && (int64_t)y < a.V ? to_f32(row[y]) : __builtin_nanf("");
}

// dL/dz of one vector: f ([j = y] - s 2^(c z - b)).
template <typename T>
__device__ __forceinline__ uint4 grad_vec(uint4 v, float c, float b, float fs, float f, int64_t j0, int64_t y) {
    float z[kVec<T>], g[kVec<T>];
    unpack<T>(v, z);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) {
        g[i] = -fs * __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], c, -b));
        if (j0 + i == y) g[i] += f;
    }
    return pack<T>(g);
}

// The gradient of elements [begin, end) of a row (begin a multiple of the vector), by the threads tid of `step`.
template <typename T>
__device__ __forceinline__ void write_grad(const T *row, T *out, int64_t begin, int64_t end, int tid, int step, float c,
                                           float b, float fs, float f, int64_t y) {
    for (int64_t j = begin + (int64_t)tid * kVec<T>; j < end; j += (int64_t)step * kVec<T>) {
        const int n = (int)(end - j < kVec<T> ? end - j : kVec<T>);
        if (n == kVec<T>) store_vec(out + j, grad_vec<T>(load_vec(row + j), c, b, fs, f, j, y));
        else store_part(out + j, grad_vec<T>(load_part(row + j, n), c, b, fs, f, j, y), n);
    }
}

template <typename T> __device__ __forceinline__ void write_zeros(T *out, int64_t begin, int64_t end, int tid, int step) {
    for (int64_t j = begin + (int64_t)tid * kVec<T>; j < end; j += (int64_t)step * kVec<T>) {
        const int n = (int)(end - j < kVec<T> ? end - j : kVec<T>);
        if (n == kVec<T>) store_vec(out + j, make_uint4(0, 0, 0, 0));
        else store_part(out + j, make_uint4(0, 0, 0, 0), n);
    }
}

// One workgroup per row.  logits and grad may be the same memory: a thread writes the elements that it has read.
template <typename T, bool GRAD> __global__ __launch_bounds__(kThreads) void policy_rows_kernel(PolicyArgs a) {
    constexpr int N = kVec<T>;
    const int64_t t = blockIdx.x;
    const T *row = reinterpret_cast<const T *>(a.logits) + t * a.ld;
    T *out = GRAD ? reinterpret_cast<T *>(a.grad) + t * a.ldg : nullptr;
    const float w = weight_of(a, t);
    if (w == 0.0f) {
        if (threadIdx.x == 0) reinterpret_cast<float4 *>(a.stats)[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (GRAD) write_zeros(out, 0, a.V, threadIdx.x, kThreads);
        return;
    }
    const int32_t y = a.targets[t];
    const float zy = target_logit(a, row, y);
    Online o{-__builtin_inff(), 0.0f, 0.0f};
    const int64_t full = a.V / N;
    int64_t i = threadIdx.x;
    for (; i + 3 * kThreads < full; i += 4 * kThreads) {
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = load_vec(row + (i + u * kThreads) * N);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float z[N];
            unpack<T>(v[u], z);
            add(o, z, a.c);
        }
    }
    for (; i < full; i += kThreads) {
        float z[N];
        unpack<T>(load_vec(row + i * N), z);
        add(o, z, a.c);
    }
    if (threadIdx.x < (unsigned)(a.V - full * N)) {
        const float z[1] = {to_f32(row[full * N + threadIdx.x])};
        add(o, z, a.c);
    }
    // fixed order: within the wave, then wave by wave
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        o = merge(o, Online{__shfl_xor(o.m, off, 64), __shfl_xor(o.mb, off, 64), __shfl_xor(o.S, off, 64)});
    __shared__ Online red[kThreads / 64];
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = o;
    __syncthreads();
    o = red[0];
    for (int k = 1; k < kThreads / 64; ++k) o = merge(o, red[k]);
    const float4 s = row_stats(a, t, w, o, zy);
    if (threadIdx.x == 0) reinterpret_cast<float4 *>(a.stats)[t] = s;
    if (GRAD) {
        const float f = s.z * a.inv_temp;
        write_grad(row, out, 0, a.V, threadIdx.x, kThreads, a.c, o.mb, f / o.S, f, y);
    }
}

// The gradient from the statistics: a workgroup per row and slice of it.
template <typename T> __global__ __launch_bounds__(kThreads) void policy_backward_kernel(PolicyArgs a, int64_t slice) {
    const int64_t t = blockIdx.x, begin = (int64_t)blockIdx.y * slice, end = begin + slice < a.V ? begin + slice : a.V;
    const T *row = reinterpret_cast<const T *>(a.logits) + t * a.ld;
    T *out = reinterpret_cast<T *>(a.grad) + t * a.ldg;
    const float lse = a.stats[4 * t + 1], slope = a.stats[4 * t + 2];
    if (slope == 0.0f) {                                   // no weight, or clipped without a KL term: nothing to read
        write_zeros(out, begin, end, threadIdx.x, kThreads);
        return;
    }
    const float f = slope * a.inv_temp * (a.grad_loss ? a.grad_loss[0] : 1.0f);
    // lse log2(e) as a rounded number and what it leaves, which joins the factor
    const float b = lse * kLog2e;
    const float rest = __builtin_fmaf(lse, kLog2e, -b) + lse * 1.925963033500e-8f;
    write_grad(row, out, begin, end, threadIdx.x, kThreads, a.c, b, f * __builtin_amdgcn_exp2f(-rest), f, a.targets[t]);
}

constexpr int kSumThreads = 1024;

// loss = sum w (surrogate + kl KL), sum w surrogate, sum w KL, sum w [outside]; FP64, fixed order.
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(PolicyArgs a) {
    double s[3] = {0.0, 0.0, 0.0};
    for (int64_t t = threadIdx.x; t < a.T; t += kSumThreads) {
        const float w = weight_of(a, t);
        if (w == 0.0f) continue;
        const float4 st = reinterpret_cast<const float4 *>(a.stats)[t];
        const float adv = a.adv[t], r = st.w;
        const float held = r < a.low ? a.low : (r > a.high ? a.high : r);
        const float x = r * adv, y = held * adv;
        s[0] += (double)w * -(double)(y < x ? y : x);
        if (a.ref) s[1] += (double)w * (double)kl_term(a.ref[t] - st.x);
        s[2] += outside(a, r, adv) ? (double)w : 0.0;
    }
    __shared__ double red[3][kSumThreads / 64];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) s[k] += __shfl_xor(s[k], off, 64);
        if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = s[k];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 0; k < 3; ++k) {
            s[k] = 0.0;
            for (int i = 0; i < kSumThreads / 64; ++i) s[k] += red[k][i];
        }
        a.loss[0] = (float)(s[0] + (double)a.kl * s[1]);
        a.loss[1] = (float)s[0];
        a.loss[2] = (float)s[1];
        a.loss[3] = (float)s[2];
    }
}

}  // namespace

hipError_t launch_policy_loss(const PolicyArgs &a, bool bf16, hipStream_t stream) {
    const dim3 grid((unsigned)a.T), block(kThreads);
    if (a.T > 0) {
        if (bf16 && a.grad) hipLaunchKernelGGL((policy_rows_kernel<uint16_t, true>), grid, block, 0, stream, a);
        else if (bf16) hipLaunchKernelGGL((policy_rows_kernel<uint16_t, false>), grid, block, 0, stream, a);
        else if (a.grad) hipLaunchKernelGGL((policy_rows_kernel<float, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((policy_rows_kernel<float, false>), grid, block, 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(kSumThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_policy_backward(const PolicyArgs &a, bool bf16, hipStream_t stream) {
    if (a.T == 0) return hipSuccess;
    // slices of a row, so that few rows give some thousand workgroups too; multiples of the workgroup's vectors
    const int64_t unit = (int64_t)kThreads * (bf16 ? 8 : 4), units = (a.V + unit - 1) / unit;
    int64_t slices = (2048 + a.T - 1) / a.T;
    slices = slices < units ? slices : units;
    const int64_t slice = (units + slices - 1) / slices * unit;
    const dim3 grid((unsigned)a.T, (unsigned)((a.V + slice - 1) / slice)), block(kThreads);
    if (bf16) hipLaunchKernelGGL(policy_backward_kernel<uint16_t>, grid, block, 0, stream, a, slice);
    else hipLaunchKernelGGL(policy_backward_kernel<float>, grid, block, 0, stream, a, slice);
    return hipGetLastError();
}

}  // namespace reqat
