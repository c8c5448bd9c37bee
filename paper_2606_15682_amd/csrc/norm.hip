// Layer norm and root-mean-square norm for gfx950, forward and backward, over rows x of K elements:
//   mu = mean x (0 unless centred),  rstd = (mean (x - mu)^2 + eps)^(-1/2),  h = (x - mu) rstd,  y = h w + b;
//   g = dy w,  dx = rstd (g - [centred] mean g - h mean(g h)),  dw = sum over rows of dy h,  db = sum over rows of dy.
//
// A row's x (and dy) stays in registers, so that the mean comes before the squares are taken, and every element is read
// once.  A group of 64, 256 or 1024 threads holds a row, VPT vectors of 16 bytes a thread; a group of 64 is one wave, four
// rows to a workgroup, without a barrier.  Groups walk over the rows in steps of the grid, the weights in registers, and in
// the backward pass each adds up its own dw and db there; a second launch joins the groups' sums in their order.
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

// Sums of N numbers over a row's group of G threads, the same in every thread.  `red` is used in turn by two halves,
// so that one barrier is enough: a half is written again only after the barrier of the other's sum.
template <int G, int N> struct GroupSum {
    static constexpr int kWaves = G / 64;
    float (*red)[N][kWaves];
    int half = 0;
    __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = wave_sum(x[k]);
        if constexpr (kWaves > 1) {
            float (*r)[kWaves] = red[half];
            half ^= 1;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) r[k][threadIdx.x >> 6] = x[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                x[k] = r[k][0];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) x[k] += r[k][w];
            }
        }
    }
};

// The group's vectors of a row: vector v of thread i holds the elements from (v G + i) kVec on.
template <typename T, int G, int VPT> __device__ __forceinline__ void load_row(const T *row, int K, int i, uint4 (&x)[VPT]) {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int j = (v * G + i) * kVec<T>, n = K - j;
        x[v] = n >= kVec<T> ? load_vec(row + j) : (n > 0 ? load_part(row + j, n) : make_uint4(0, 0, 0, 0));
    }
}

template <typename T> __device__ __forceinline__ void store_at(T *row, int K, int j, const float (&z)[kVec<T>]) {
    const int n = K - j;
    if (n >= kVec<T>) store_vec(row + j, pack<T>(z));
    else if (n > 0) store_part(row + j, pack<T>(z), n);
}

// Parameters of the thread's elements as FP32; zero where there is no parameter or no element.
template <typename T, int G, int VPT>
__device__ __forceinline__ void load_params(const void *w, bool bf16, int K, int i, float (&out)[VPT][kVec<T>]) {
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) {
            const int j = (v * G + i) * kVec<T> + e;
            out[v][e] = 0.0f;
            if (w && j < K) out[v][e] = bf16 ? to_f32(reinterpret_cast<const uint16_t *>(w)[j]) : reinterpret_cast<const float *>(w)[j];
        }
}

template <typename T, int G, int VPT>
__global__ __launch_bounds__(G == 64 ? 256 : G) void norm_forward_kernel(NormArgs a) {
    constexpr int N = kVec<T>, kRows = G == 64 ? 4 : 1;
    __shared__ float red[2][1][G / 64];
    GroupSum<G, 1> sum{red};
    const int i = G == 64 ? (threadIdx.x & 63) : threadIdx.x;
    const int K = (int)a.K;
    const float inv = 1.0f / (float)K;
    float w[VPT][N], b[VPT][N];
    load_params<T, G, VPT>(a.w, a.w_bf16, K, i, w);
    load_params<T, G, VPT>(a.b, a.w_bf16, K, i, b);
    for (int64_t r = (int64_t)blockIdx.x * kRows + (G == 64 ? threadIdx.x >> 6 : 0); r < a.M; r += (int64_t)gridDim.x * kRows) {
        uint4 raw[VPT];
        load_row<T, G, VPT>(reinterpret_cast<const T *>(a.x) + r * a.ldx, K, i, raw);
        float x[VPT][N], s[1] = {0.0f}, mu = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) unpack<T>(raw[v], x[v]);
        if (a.center) {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int e = 0; e < N; ++e) s[0] += x[v][e];
            sum(s);
            mu = s[0] * inv;
        }
        s[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[v][e] -= mu;
                const bool in = (v * G + i) * N + e < K;
                s[0] = __builtin_fmaf(in ? x[v][e] : 0.0f, x[v][e], s[0]);
            }
        sum(s);
        const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
        T *y = reinterpret_cast<T *>(a.y) + r * a.ldy;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[v][e] = __builtin_fmaf(x[v][e] * rstd, w[v][e], b[v][e]);
            store_at(y, K, (v * G + i) * N, x[v]);
        }
        if (i == 0) {
            a.stats[2 * r] = mu;
            a.stats[2 * r + 1] = rstd;
        }
    }
}

template <typename T, int G, int VPT>
__global__ __launch_bounds__(G == 64 ? 256 : G) void norm_backward_kernel(NormArgs a) {
    constexpr int N = kVec<T>, kRows = G == 64 ? 4 : 1;
    __shared__ float red[2][2][G / 64];
    GroupSum<G, 2> sum{red};
    const int i = G == 64 ? (threadIdx.x & 63) : threadIdx.x;
    const int K = (int)a.K;
    const float inv = 1.0f / (float)K;
    float w[VPT][N], dw[VPT][N] = {}, db[VPT][N] = {};
    load_params<T, G, VPT>(a.w, a.w_bf16, K, i, w);
    const int64_t group = (int64_t)blockIdx.x * kRows + (G == 64 ? threadIdx.x >> 6 : 0), groups = (int64_t)gridDim.x * kRows;
    for (int64_t r = group; r < a.M; r += groups) {
        uint4 xr[VPT], yr[VPT];
        load_row<T, G, VPT>(reinterpret_cast<const T *>(a.x) + r * a.ldx, K, i, xr);
        load_row<T, G, VPT>(reinterpret_cast<const T *>(a.dy) + r * a.lddy, K, i, yr);
        const float mu = a.center ? a.stats[2 * r] : 0.0f, rstd = a.stats[2 * r + 1];
        float s[2] = {0.0f, 0.0f};                      // sum g, sum g h; zeros beyond K: dy and w are zero there
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float x[N], dy[N];
            unpack<T>(xr[v], x);
            unpack<T>(yr[v], dy);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float h = (x[e] - mu) * rstd, g = dy[e] * w[v][e];
                s[0] += g;
                s[1] = __builtin_fmaf(g, h, s[1]);
                dw[v][e] = __builtin_fmaf(dy[e], h, dw[v][e]);
                db[v][e] += dy[e];
            }
        }
        sum(s);
        const float c0 = a.center ? s[0] * inv : 0.0f, c1 = s[1] * inv;
        T *dx = reinterpret_cast<T *>(a.dx) + r * a.lddx;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float x[N], dy[N];
            unpack<T>(xr[v], x);
            unpack<T>(yr[v], dy);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float h = (x[e] - mu) * rstd;
                x[e] = rstd * (__builtin_fmaf(dy[e], w[v][e], -c0) - h * c1);
            }
            store_at(dx, K, (v * G + i) * N, x);
        }
    }
    float *part = a.partials + group * K;
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int j = (v * G + i) * N + e;
            if (j < K) {
                part[j] = dw[v][e];
                if (a.db) part[groups * K + j] = db[v][e];
            }
        }
}

// dw (blockIdx.y 0) and db (1): 64 columns a workgroup, the groups' sums in 16 strips, the strips in turn.
__global__ __launch_bounds__(1024) void norm_params_kernel(NormArgs a, int64_t groups) {
    const int64_t j = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int strip = threadIdx.x >> 6;
    const float *part = a.partials + (int64_t)blockIdx.y * groups * a.K;
    float s = 0.0f;
    if (j < a.K) {
#pragma unroll 8
        for (int64_t g = strip; g < groups; g += 16) s += part[g * a.K + j];
    }
    __shared__ float red[16][64];
    red[strip][threadIdx.x & 63] = s;
    __syncthreads();
    if (strip == 0 && j < a.K) {
        for (int k = 1; k < 16; ++k) s += red[k][threadIdx.x];
        void *out = blockIdx.y ? a.db : a.dw;
        if (a.w_bf16) reinterpret_cast<uint16_t *>(out)[j] = from_f32<uint16_t>(s);
        else reinterpret_cast<float *>(out)[j] = s;
    }
}

template <typename T, int G> hipError_t launch(const NormArgs &a, int vpt, bool backward, dim3 grid, hipStream_t stream) {
    const dim3 block(G == 64 ? 256 : G);
#define REQAT_NORM(V)                                                                                                  \
    case V:                                                                                                            \
        if (backward) hipLaunchKernelGGL((norm_backward_kernel<T, G, V>), grid, block, 0, stream, a);                  \
        else hipLaunchKernelGGL((norm_forward_kernel<T, G, V>), grid, block, 0, stream, a);                            \
        break;
    switch (vpt) {
        REQAT_NORM(1)
        REQAT_NORM(2)
        REQAT_NORM(3)
        REQAT_NORM(4)
    default:
        if constexpr (G == 1024 && sizeof(T) == 4) {
            switch (vpt) {
                REQAT_NORM(5)
                REQAT_NORM(6)
                REQAT_NORM(7)
                REQAT_NORM(8)
            }
        }
    }
#undef REQAT_NORM
    return hipGetLastError();
}

template <typename T> hipError_t launch_typed(const NormArgs &a, bool backward, hipStream_t stream) {
    const NormPlan p = norm_plan(a.M, a.K, sizeof(T) == 2);
    const dim3 grid((unsigned)p.workgroups);
    const hipError_t e = a.M == 0 ? hipSuccess           // no rows: zeros from no groups
                         : p.threads == 64 ? launch<T, 64>(a, p.vpt, backward, grid, stream)
                         : p.threads == 256 ? launch<T, 256>(a, p.vpt, backward, grid, stream)
                                            : launch<T, 1024>(a, p.vpt, backward, grid, stream);
    if (e != hipSuccess || !backward) return e;
    hipLaunchKernelGGL(norm_params_kernel, dim3((unsigned)((a.K + 63) / 64), a.db ? 2 : 1), dim3(1024), 0, stream, a, p.groups);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, bool bf16, bool backward, hipStream_t stream) {
    return bf16 ? launch_typed<uint16_t>(a, backward, stream) : launch_typed<float>(a, backward, stream);
}

}  // namespace reqat
