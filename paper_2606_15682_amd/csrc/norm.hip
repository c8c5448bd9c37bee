// Layer norm and root-mean-square norm for gfx950, forward and backward, over rows x of K elements:
//   mu = mean x (0 unless centred),  rstd = (mean (x - mu)^2 + eps)^(-1/2),  h = (x - mu) rstd,  y = h w + b;
//   g = dy w,  dx = rstd (g - [centred] mean g - h mean(g h)),  dw = sum over rows of dy h,  db = sum over rows of dy.
//
// A row's x (and dy) stays in registers, so that the mean comes before the squares are taken, and every element is read
// once.  A group of 64, 256, 512 or 1024 threads holds a row, VPT vectors of 16 bytes a thread; a group of 64 is one wave,
// four of them to a workgroup, without a barrier.  Groups walk over the rows in steps of the grid, the weights in registers.
// In the backward pass each adds up its own dw and db there and asks for its next row before it works on one; the groups
// of a workgroup join theirs through LDS, and a second launch joins the workgroups' in their order.  Rows of more than four
// vectors a thread leave no registers for dw and db: a launch of its own adds them up by columns.
//
// Forward at the rate of a large copy (9001 x 3584 bfloat16 24 us, 5.4 TB/s), backward too up to 12288 bfloat16 elements a row
// (8192 x 5120 46 + 5 us, 5.0 TB/s).  Rows of 12289 to 16384 spill 25 registers backward (4096 x 13824: 102 us for the 66 of a copy),
// FP32 rows of more than 20480 elements 5 to 22, and the columns' pass reads x and dy once more (2048 x 27648: 137 us for 66).
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

// Sums of N numbers over a row's group of G threads, the same in every thread; group g of the workgroup's P.  `red` is used
// in turn by two halves, so that one barrier is enough: a half is written again only after the barrier of the other's sum.
template <int G, int P, int N> struct GroupSum {
    static constexpr int kWaves = G / 64;
    float (*red)[P][N][kWaves];
    int g, half = 0;
    __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = wave_sum(x[k]);
        if constexpr (kWaves > 1) {
            float (*r)[kWaves] = red[half][g];
            half ^= 1;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) r[k][(threadIdx.x % G) >> 6] = x[k];
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

// N parameters from element j on, n of them exist; zeros behind them.
template <typename W, int N> __device__ __forceinline__ void load_params_of(const W *w, int n, float (&out)[N]) {
    W e[N] = {};
    if (n >= N) {
        __builtin_memcpy(e, w, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) e[i] = w[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = to_f32(e[i]);
}

// Parameters from element j on as FP32; zero where there is no parameter or no element.
template <int N> __device__ __forceinline__ void load_params_at(const void *w, bool bf16, int K, int j, float (&out)[N]) {
    const int n = w ? K - j : 0;
    if (bf16) load_params_of(reinterpret_cast<const uint16_t *>(w) + j, n, out);
    else load_params_of(reinterpret_cast<const float *>(w) + j, n, out);
}

// Where a thread's vectors of a row of K >= kVec elements lie, so that every access is a whole vector and none stands
// behind a branch, where the compiler waits for all loads in flight.  The last vector of a row whose length is no multiple of
// it ends with the row: its first `skip` elements are the vector's before it once more, get the same results in both
// places, and count in the sums once.  A thread without elements there reads the row's first vector; all its elements are
// skipped and nothing of it is written.  (All vectors but a thread's last are whole: the group's last step is not full only
// there.)
template <typename T, int G, int VPT> struct Places {
    int i, at_last, skip;
    bool last;
    __device__ __forceinline__ Places(int i, int K) : i(i) {
        constexpr int N = kVec<T>;
        const int start = ((VPT - 1) * G + i) * N;
        last = start < K;
        at_last = last ? (start < K - N ? start : K - N) : 0;
        skip = last ? start - at_last : N;
    }
    __device__ __forceinline__ int at(int v) const { return v < VPT - 1 ? (v * G + i) * kVec<T> : at_last; }
    __device__ __forceinline__ bool mine(int v) const { return v < VPT - 1 || last; }
    __device__ __forceinline__ bool counts(int v, int e) const { return v < VPT - 1 || e >= skip; }
};

// The thread's parameters.  WHOLE: the row has at least a vector.
template <typename T, int G, int VPT, bool WHOLE>
__device__ __forceinline__ void load_params(const void *w, bool bf16, int K, const Places<T, G, VPT> &p, float (&out)[VPT][kVec<T>]) {
    constexpr int N = kVec<T>;
    if (!WHOLE || !w) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) load_params_at(w, bf16, K, (v * G + p.i) * N, out[v]);
    } else if (bf16) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) load_params_of(reinterpret_cast<const uint16_t *>(w) + p.at(v), N, out[v]);
    } else {
#pragma unroll
        for (int v = 0; v < VPT; ++v) load_params_of(reinterpret_cast<const float *>(w) + p.at(v), N, out[v]);
    }
}

__device__ __forceinline__ uint4 where(bool in, uint4 v) {
    return make_uint4(in ? v.x : 0, in ? v.y : 0, in ? v.z : 0, in ? v.w : 0);
}

template <int N> __device__ __forceinline__ void put_sums(float *p, int n, const float (&z)[N]) {
    if (n >= N) {
        __builtin_memcpy(p, z, sizeof(z));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < n) p[e] = z[e];
    }
}

template <typename T, int G, int VPT, bool WHOLE>
__global__ __launch_bounds__(G == 64 ? 256 : G) void norm_forward_kernel(NormArgs a) {
    constexpr int N = kVec<T>, kRows = G == 64 ? 4 : 1;
    __shared__ float red[2][1][1][G / 64];
    GroupSum<G, 1, 1> sum{red, 0};
    const int i = threadIdx.x % G;
    const int K = (int)a.K;
    const float inv = 1.0f / (float)K;
    const Places<T, G, VPT> p(i, K);
    float w[VPT][N], b[VPT][N];
    load_params<T, G, VPT, WHOLE>(a.w, a.w_bf16, K, p, w);
    load_params<T, G, VPT, WHOLE>(a.b, a.w_bf16, K, p, b);
    for (int64_t r = (int64_t)blockIdx.x * kRows + (G == 64 ? threadIdx.x >> 6 : 0); r < a.M; r += (int64_t)gridDim.x * kRows) {
        uint4 raw[VPT];
        const T *row = reinterpret_cast<const T *>(a.x) + r * a.ldx;
        if constexpr (WHOLE) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) raw[v] = load_vec(row + p.at(v));
        } else {
            load_row<T, G, VPT>(row, K, i, raw);
        }
        float x[VPT][N], s[1] = {0.0f}, mu = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) unpack<T>(raw[v], x[v]);
        if (a.center) {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int e = 0; e < N; ++e) s[0] += !WHOLE || p.counts(v, e) ? x[v][e] : 0.0f;
            sum(s);
            mu = s[0] * inv;
        }
        s[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[v][e] -= mu;
                const bool in = WHOLE ? p.counts(v, e) : (v * G + i) * N + e < K;
                const float d = in ? x[v][e] : 0.0f;    // both factors: an element read once more may be infinite
                s[0] = __builtin_fmaf(d, d, s[0]);
            }
        sum(s);
        const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
        T *y = reinterpret_cast<T *>(a.y) + r * a.ldy;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[v][e] = __builtin_fmaf(x[v][e] * rstd, w[v][e], b[v][e]);
            if constexpr (WHOLE) {
                if (p.mine(v)) store_vec(y + p.at(v), pack<T>(x[v]));
            } else {
                store_at(y, K, (v * G + i) * N, x[v]);
            }
        }
        if (i == 0) {
            a.stats[2 * r] = mu;
            a.stats[2 * r + 1] = rstd;
        }
    }
}

// The vector as it came, after x is known: keeps the compiler from unpacking all vectors first, or from holding them unpacked
// from the sums to dx, in two or four times the registers.
__device__ __forceinline__ void pin(uint4 &v, float x) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w) : "v"(x)); }

// WHOLE: the row has at least a vector, and Places says where the thread's are.
template <typename T, int G, int VPT, bool WHOLE>
__global__ __launch_bounds__(G *norm_groups(G)) void norm_backward_kernel(NormArgs a) {
    constexpr int N = kVec<T>, P = norm_groups(G);
    // up to four vectors: the weights and the sums of dw and db in registers, and a row ahead; else dx alone, the weights
    // read for every row
    constexpr bool kHold = VPT <= 4;
    __shared__ float red[2][P][2][G / 64];
    const int i = threadIdx.x % G, g = threadIdx.x / G, K = (int)a.K;
    GroupSum<G, P, 2> sum{red, g};
    const float inv = 1.0f / (float)K;
    constexpr int kSums = kHold ? VPT : 1;
    float held[kSums][N], dw[kSums][N] = {}, db[kSums][N] = {};
    const Places<T, G, VPT> p(i, K);
    if constexpr (kHold) load_params<T, G, VPT, WHOLE>(a.w, a.w_bf16, K, p, held);
    uint4 xr[VPT], yr[VPT];
    float2 sr;                                          // mean and 1 / deviation of the row in xr
    const auto load = [&](int64_t r) {                  // a row behind the last one: zeros, which add nothing
        const bool in = r < a.M;
        __builtin_memcpy(&sr, a.stats + 2 * (in ? r : 0), 8);
        const T *x = reinterpret_cast<const T *>(a.x) + (in ? r : 0) * a.ldx;
        const T *dy = reinterpret_cast<const T *>(a.dy) + (in ? r : 0) * a.lddy;
        if constexpr (WHOLE) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                xr[v] = load_vec(x + p.at(v));
                yr[v] = load_vec(dy + p.at(v));
            }
        } else {
            load_row<T, G, VPT>(x, in ? K : 0, i, xr);
            load_row<T, G, VPT>(dy, in ? K : 0, i, yr);
        }
    };
    // all groups of a workgroup take the same number of turns
    const int64_t step = (int64_t)gridDim.x * P;
    load((int64_t)blockIdx.x * P + g);
    for (int64_t r0 = (int64_t)blockIdx.x * P; r0 < a.M; r0 += step) {
        const int64_t r = r0 + g;
        const bool in = r < a.M;
        const float mu = a.center && in ? sr.x : 0.0f, rstd = in ? sr.y : 0.0f;
        uint4 x0[VPT], y0[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            x0[v] = WHOLE && P > 1 ? where(in, xr[v]) : xr[v];      // with one group a workgroup, every row is one
            y0[v] = WHOLE && P > 1 ? where(in, yr[v]) : yr[v];
        }
        if (kHold) load(r + step);
        float s[2] = {0.0f, 0.0f};                      // sum g, sum g h; zeros beyond K: dy and w are zero there
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float x[N], dy[N], w[N];
            if (!kHold) pin(x0[v], s[1]);
            unpack<T>(x0[v], x);
            unpack<T>(y0[v], dy);
            if constexpr (!kHold) load_params_at(a.w, a.w_bf16, K, WHOLE ? p.at(v) : (v * G + i) * N, w);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if constexpr (kHold) w[e] = held[v][e];
                const bool counts = !WHOLE || p.counts(v, e);
                const float h = (x[e] - mu) * rstd, gr = counts ? dy[e] * w[e] : 0.0f;
                s[0] += gr;
                s[1] = __builtin_fmaf(gr, counts ? h : 0.0f, s[1]);
                if constexpr (kHold) {
                    dw[v][e] = __builtin_fmaf(dy[e], h, dw[v][e]);
                    db[v][e] += dy[e];
                }
            }
        }
        sum(s);
        const float c0 = a.center ? s[0] * inv : 0.0f, c1 = s[1] * inv;
        T *dx = reinterpret_cast<T *>(a.dx) + r * a.lddx;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            pin(x0[v], c1);
            pin(y0[v], c1);
            float x[N], dy[N], w[N];
            unpack<T>(x0[v], x);
            unpack<T>(y0[v], dy);
            if constexpr (!kHold) load_params_at(a.w, a.w_bf16, K, WHOLE ? p.at(v) : (v * G + i) * N, w);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if constexpr (kHold) w[e] = held[v][e];
                const float h = (x[e] - mu) * rstd;
                x[e] = rstd * (__builtin_fmaf(dy[e], w[e], -c0) - h * c1);
            }
            if constexpr (WHOLE) {
                if (in && p.mine(v)) store_vec(dx + p.at(v), pack<T>(x));
            } else {
                store_at(dx, in ? K : 0, (v * G + i) * N, x);
            }
        }
        if (!kHold) load(r + step);
    }
    if constexpr (!kHold) return;
    // the groups' sums, the second's and further ones to the first's
    extern __shared__ float others[];                   // [K] of dw, then of db
#pragma unroll
    for (int from = 1; from < P; ++from) {
        __syncthreads();
        if (g == from) {
#pragma unroll
            for (int v = 0; v < kSums; ++v) {
                const int j = WHOLE ? p.at(v) : (v * G + i) * N;
                if (WHOLE ? p.mine(v) : j < K) {
                    put_sums(others + j, K - j, dw[v]);
                    put_sums(others + K + j, K - j, db[v]);
                }
            }
        }
        __syncthreads();
        if (g == 0) {
#pragma unroll
            for (int v = 0; v < kSums; ++v) {
                const int j = WHOLE ? p.at(v) : (v * G + i) * N;
                if (WHOLE ? p.mine(v) : j < K) {
                    float x[N], y[N];
                    load_params_of(others + j, K - j, x);
                    load_params_of(others + K + j, K - j, y);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        dw[v][e] += x[e];
                        db[v][e] += y[e];
                    }
                }
            }
        }
    }
    if (g > 0) return;
    float *part = a.partials + (int64_t)blockIdx.x * K;
#pragma unroll
    for (int v = 0; v < kSums; ++v)
        if (WHOLE ? p.mine(v) : (v * G + i) * N < K) {
            const int j = WHOLE ? p.at(v) : (v * G + i) * N;
            put_sums(part + j, K - j, dw[v]);
            if (a.db) put_sums(part + (int64_t)gridDim.x * K + j, K - j, db[v]);
        }
}

// dw and db by columns: 256 vectors of them (blockIdx.x), over the rows of part blockIdx.y.
template <typename T> __global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a, int64_t rows) {
    constexpr int N = kVec<T>, U = 4;
    const int K = (int)a.K, j = ((int)blockIdx.x * 256 + (int)threadIdx.x) * N, n = K - j;
    if (n <= 0) return;
    const int64_t begin = (int64_t)blockIdx.y * rows, end = begin + rows < a.M ? begin + rows : a.M;
    const T *x = reinterpret_cast<const T *>(a.x) + j, *dy = reinterpret_cast<const T *>(a.dy) + j;
    float dw[N] = {}, db[N] = {};
    for (int64_t r0 = begin; r0 < end; r0 += U) {
        uint4 xr[U], yr[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t r = r0 + u < end ? r0 + u : end - 1;
            xr[u] = n >= N ? load_vec(x + r * a.ldx) : load_part(x + r * a.ldx, n);
            yr[u] = n >= N ? load_vec(dy + r * a.lddy) : load_part(dy + r * a.lddy, n);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + u >= end) break;
            const float mu = a.center ? a.stats[2 * (r0 + u)] : 0.0f, rstd = a.stats[2 * (r0 + u) + 1];
            float xv[N], yv[N];
            unpack<T>(xr[u], xv);
            unpack<T>(yr[u], yv);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                dw[e] = __builtin_fmaf(yv[e], (xv[e] - mu) * rstd, dw[e]);
                db[e] += yv[e];
            }
        }
    }
    float *part = a.partials + (int64_t)blockIdx.y * K + j;
    put_sums(part, n, dw);
    if (a.db) put_sums(part + (int64_t)gridDim.y * K, n, db);
}

// dw (blockIdx.y 0) and db (1): 64 columns a workgroup, the workgroups' sums in 16 strips, the strips in turn.
__global__ __launch_bounds__(1024) void norm_params_kernel(NormArgs a, int64_t parts) {
    const int64_t j = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int strip = threadIdx.x >> 6;
    const float *part = a.partials + (int64_t)blockIdx.y * parts * a.K;
    float s = 0.0f;
    if (j < a.K) {
#pragma unroll 8
        for (int64_t g = strip; g < parts; g += 16) s += part[g * a.K + j];
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

// The kernel of G threads and V vectors each, or of fewer, down to the fewest that norm_plan gives G threads.
template <typename T, int G, int V = norm_most_vectors(G)>
hipError_t launch(const NormArgs &a, const NormPlan &p, bool backward, hipStream_t stream) {
    if constexpr (V > norm_least_vectors(G)) {
        if (p.vpt < V) return launch<T, G, V - 1>(a, p, backward, stream);
    }
    if (p.vpt != V) return hipErrorInvalidValue;
    constexpr int P = norm_groups(G);
    const dim3 grid((unsigned)(backward ? p.backward : p.forward)), forward(G == 64 ? 256 : G);
    const size_t lds = P > 1 ? (size_t)a.K * 8 : 0;
    if constexpr (G == 64 && V == 1) {                   // the one form for rows of less than a vector
        if (a.K < kVec<T>) {
            if (backward) hipLaunchKernelGGL((norm_backward_kernel<T, G, V, false>), grid, dim3(G * P), lds, stream, a);
            else hipLaunchKernelGGL((norm_forward_kernel<T, G, V, false>), grid, forward, 0, stream, a);
            return hipGetLastError();
        }
    }
    if (backward) hipLaunchKernelGGL((norm_backward_kernel<T, G, V, true>), grid, dim3(G * P), lds, stream, a);
    else hipLaunchKernelGGL((norm_forward_kernel<T, G, V, true>), grid, forward, 0, stream, a);
    return hipGetLastError();
}

// More than 4096 vectors: FP32 alone.
template <typename T> hipError_t launch_widest(const NormArgs &a, const NormPlan &p, bool backward, hipStream_t stream) {
    if constexpr (sizeof(T) == 4) return launch<T, 1024>(a, p, backward, stream);
    return hipErrorInvalidValue;
}

template <typename T> hipError_t launch_typed(const NormArgs &a, bool backward, hipStream_t stream) {
    const NormPlan p = norm_plan(a.M, a.K, sizeof(T) == 2);
    if (backward && p.columns && a.M > 0) {              // before dx, which may take the place of x or dy
        const int64_t tile = 256 * kVec<T>;
        hipLaunchKernelGGL(norm_columns_kernel<T>, dim3((unsigned)((a.K + tile - 1) / tile), (unsigned)p.sums), dim3(256), 0, stream, a,
                           (a.M + p.sums - 1) / p.sums);
        const hipError_t c = hipGetLastError();
        if (c != hipSuccess) return c;
    }
    const hipError_t e = a.M == 0 ? hipSuccess           // no rows: zeros from no sums
                         : p.threads == 64 ? launch<T, 64>(a, p, backward, stream)
                         : p.threads == 256 ? launch<T, 256>(a, p, backward, stream)
                         : p.threads == 512 ? launch<T, 512>(a, p, backward, stream)
                                            : launch_widest<T>(a, p, backward, stream);
    if (e != hipSuccess || !backward) return e;
    hipLaunchKernelGGL(norm_params_kernel, dim3((unsigned)((a.K + 63) / 64), a.db ? 2 : 1), dim3(1024), 0, stream, a, p.sums);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, bool bf16, bool backward, hipStream_t stream) {
    return bf16 ? launch_typed<uint16_t>(a, backward, stream) : launch_typed<float>(a, backward, stream);
}

}  // namespace reqat
