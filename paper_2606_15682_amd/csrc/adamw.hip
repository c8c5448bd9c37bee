// AdamW over many tensors for gfx950, states in FP32 or in 8 bits.  Per element, every operation rounded to FP32:
//   g = grad [grad_scale],  m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,  u = sqrt(v'),
//   p' = decay p - step (m' / (root u + eps)),   decay = 1 - lr wd, step = lr / (1 - b1^t), root = (1 - b2^t)^(-1/2).
// 8-bit states go in blocks of 128 elements of a tensor, each with an FP32 scale: m as E4M3 of m / s, s = max |m| / 448;
// v as its root u, in 8 bits without a sign, 2^-15 (1 + 1/16) .. 1.9375 with four bits behind the binary point, of u / s,
// s = max u / 1.9375.  The parameter's step takes m' and u before they are rounded.
//
// The tensors' addresses travel in the kernel's arguments, kBatch tensors to a launch, so nothing is copied and a step can
// be captured.  A workgroup does kChunk elements of one tensor, found by bisection over the tensors' first workgroups.
//
// Bound by memory: 275 million elements with FP32 states, bfloat16 gradients and copies in 1429 us, 5.4 TB/s of 28 bytes an
// element (runs of 4096 elements a workgroup 1447 us, of 8192 1461 us; stores through the caches 1455 us).  8-bit states:
// 60 million elements of one tensor in 217 us, 4.4 TB/s of 16 bytes, half of it vector instructions: three exact divisions
// and a root an element, without which it takes 186 us but the codes would not be those of the rule.
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

constexpr int kThreads = 256, kSteps = 2, kChunk = kThreads * 4 * kSteps;
constexpr int kBatch = 56;
constexpr uint32_t kInf = 0x7F800000u;

struct Batch {
    AdamTensor tensor[kBatch];
    uint32_t first[kBatch + 1];                         // first workgroup of a tensor
    int32_t count;
    AdamCoef c;
    const float *dev_coef, *grad_scale;
};
static_assert(sizeof(Batch) <= 4096, "kernel arguments");

// Four elements from p on, n of them exist (n <= 0: none); zeros for the others.
template <typename T> __device__ __forceinline__ void load4(const T *p, int64_t n, float (&z)[4]) {
    T e[4] = {T(0), T(0), T(0), T(0)};
    if (n >= 4) {
        __builtin_memcpy(e, p, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) e[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = to_f32(e[i]);
}

// Written past the caches: a step's results are not read again before the next step.
template <typename T> __device__ __forceinline__ void store4(T *p, int64_t n, const float (&z)[4]) {
    typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    T e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = from_f32<T>(z[i]);
    if (n >= 4) {
        __builtin_nontemporal_store((Four){e[0], e[1], e[2], e[3]}, reinterpret_cast<Four *>(p));
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) p[i] = e[i];
    }
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int64_t n) {
    uint32_t w = 0;
    if (n >= 4) __builtin_memcpy(&w, p, 4);
    else
        for (int i = 0; i < 3; ++i)
            if (i < n) w |= (uint32_t)p[i] << (8 * i);
    return w;
}

__device__ __forceinline__ void store_codes(uint8_t *p, int64_t n, uint32_t w) {
    if (n >= 4) __builtin_memcpy(p, &w, 4);
    else
        for (int i = 0; i < 3; ++i)
            if (i < n) p[i] = (uint8_t)(w >> (8 * i));
}

__device__ __forceinline__ void values_m(uint32_t w, float s, float (&m)[4]) {
    m[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * s;
    m[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * s;
    m[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * s;
    m[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * s;
}

__device__ __forceinline__ void values_u(uint32_t w, float s, float (&u)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = (w >> (8 * i)) & 255u;
        u[i] = c ? __uint_as_float((c + 0x700u) << 19) * s : 0.0f * s;
    }
}

// Largest magnitude pattern of the block's 128 elements, four of them in each of 32 lanes.
__device__ __forceinline__ uint32_t block_max(const float (&z)[4]) {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = __float_as_uint(z[i]) & 0x7FFFFFFFu;
        x = b > x ? b : x;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const uint32_t b = (uint32_t)__shfl_xor((int)x, off, 64);
        x = b > x ? b : x;
    }
    return x;
}

// The block's scale: NaN for a block with NaN or Inf, whose codes are 0 then.
__device__ __forceinline__ float block_scale(uint32_t max, float top) {
    return max >= kInf ? __builtin_nanf("") : __uint_as_float(max) / top;
}

__device__ __forceinline__ uint32_t codes_m(const float (&m)[4], float s) {
    if (!(s > 0.0f)) return 0;
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_fminf(__builtin_fmaxf(m[i] / s, -448.0f), 448.0f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
}

__device__ __forceinline__ uint32_t codes_u(const float (&u)[4], float s) {
    if (!(s > 0.0f)) return 0;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = u[i] / s;
        const uint32_t b = __float_as_uint(x);
        int c = (int)((b + 0x3FFFFu + ((b >> 19) & 1u)) >> 19) - 0x700;
        c = c < 1 ? 1 : (c > 255 ? 255 : c);
        w |= (x > 0.0f ? (uint32_t)c : 0u) << (8 * i);
    }
    return w;
}

// The batch's tensor of workgroup b: the last one whose first workgroup is not behind b.
__device__ __forceinline__ int find(const Batch &a, uint32_t b) {
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= b) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename P, typename G, int BITS> __global__ __launch_bounds__(kThreads) void adamw_kernel(const Batch a) {
    const int k = find(a, blockIdx.x);
    const AdamTensor t = a.tensor[k];
    const int64_t at = (int64_t)(blockIdx.x - a.first[k]) * kChunk + threadIdx.x * 4;
    P *p = reinterpret_cast<P *>(t.p) + at;
    const G *g = reinterpret_cast<const G *>(t.g) + at;
    const float gs = a.grad_scale ? a.grad_scale[0] : 1.0f;
    AdamCoef c = a.c;
    if (a.dev_coef) {
        c.decay = a.dev_coef[0];
        c.step = a.dev_coef[1];
        c.root = a.dev_coef[2];
    }
    float pv[kSteps][4], gv[kSteps][4], mv[kSteps][4], vv[kSteps][4];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t o = (int64_t)s * kThreads * 4, n = t.n - at - o;
        load4(p + o, n, pv[s]);
        load4(g + o, n, gv[s]);
        if constexpr (BITS == 32) {
            load4(reinterpret_cast<const float *>(t.m) + at + o, n, mv[s]);
            load4(reinterpret_cast<const float *>(t.v) + at + o, n, vv[s]);
        } else {
            const int64_t b = (at + o) / kAdamBlock;
            values_m(load_codes(reinterpret_cast<const uint8_t *>(t.m) + at + o, n), n > 0 ? t.m_scale[b] : 0.0f, mv[s]);
            values_u(load_codes(reinterpret_cast<const uint8_t *>(t.v) + at + o, n), n > 0 ? t.v_scale[b] : 0.0f, vv[s]);
        }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t o = (int64_t)s * kThreads * 4, n = t.n - at - o;
        float u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float grad = gv[s][i] * gs;
            if constexpr (BITS == 8) vv[s][i] *= vv[s][i];
            mv[s][i] = c.b1 * mv[s][i] + c.c1 * grad;
            vv[s][i] = c.b2 * vv[s][i] + c.c2 * (grad * grad);
            u[i] = sqrtf(vv[s][i]);
            pv[s][i] = c.decay * pv[s][i] - c.step * (mv[s][i] / (c.root * u[i] + c.eps));
        }
        store4(p + o, n, pv[s]);
        if (t.copy) store4(reinterpret_cast<uint16_t *>(t.copy) + at + o, n, pv[s]);
        if constexpr (BITS == 32) {
            store4(reinterpret_cast<float *>(t.m) + at + o, n, mv[s]);
            store4(reinterpret_cast<float *>(t.v) + at + o, n, vv[s]);
        } else {
            // elements beyond the tensor are zeros (their states and gradients were read as zeros)
            const float sm = block_scale(block_max(mv[s]), 448.0f), sv = block_scale(block_max(u), 1.9375f);
            store_codes(reinterpret_cast<uint8_t *>(t.m) + at + o, n, codes_m(mv[s], sm));
            store_codes(reinterpret_cast<uint8_t *>(t.v) + at + o, n, codes_u(u, sv));
            if (n > 0 && (threadIdx.x & 31) == 0) {
                const int64_t b = (at + o) / kAdamBlock;
                t.m_scale[b] = sm;
                t.v_scale[b] = sv;
            }
        }
    }
}

// The step's number and factors on the device: *step counts up, so that a captured step moves on with every replay.
__global__ void adamw_coef_kernel(double lr, double beta1, double beta2, double decay, const float *lr_dev, int32_t *step,
                                  float *coef) {
    const int32_t t = step[0] + 1;
    step[0] = t;
    const double rate = lr_dev ? (double)lr_dev[0] : lr;
    coef[0] = (float)(1.0 - rate * decay);
    coef[1] = (float)(rate / -expm1((double)t * log(beta1)));
    coef[2] = (float)(1.0 / sqrt(-expm1((double)t * log(beta2))));
}

// Values of 8-bit states: m = code s, v = (code s)^2.
__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(const uint8_t *mc, const float *ms, const uint8_t *vc,
                                                                 const float *vs, int64_t n, float *m, float *v) {
    const int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4, left = n - at;
    if (left <= 0) return;
    float x[4], u[4];
    values_m(load_codes(mc + at, left), ms[at / kAdamBlock], x);
    values_u(load_codes(vc + at, left), vs[at / kAdamBlock], u);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] *= u[i];
    store4(m + at, left, x);
    store4(v + at, left, u);
}

template <typename P, typename G> void launch_batch(const Batch &b, int bits, hipStream_t stream) {
    const dim3 grid(b.first[b.count]), block(kThreads);
    if (bits == 32) hipLaunchKernelGGL((adamw_kernel<P, G, 32>), grid, block, 0, stream, b);
    else hipLaunchKernelGGL((adamw_kernel<P, G, 8>), grid, block, 0, stream, b);
}

}  // namespace

hipError_t launch_adamw(const AdamTensor *tensors, int64_t count, bool p_bf16, bool g_bf16, int bits, const AdamCoef &c,
                        const float *dev_coef, const float *grad_scale, hipStream_t stream) {
    Batch b;
    b.c = c;
    b.dev_coef = dev_coef;
    b.grad_scale = grad_scale;
    b.count = 0;
    b.first[0] = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (tensors[i].n > 0) {
            b.tensor[b.count] = tensors[i];
            b.first[b.count + 1] = b.first[b.count] + (uint32_t)((tensors[i].n + kChunk - 1) / kChunk);
            ++b.count;
        }
        // a launch has fewer than 2^24 workgroups (2^32 threads)
        const uint64_t next = i + 1 < count ? (uint64_t)((tensors[i + 1].n + kChunk - 1) / kChunk) : 0;
        if (b.count > 0 && (b.count == kBatch || i + 1 == count || b.first[b.count] + next >= (1u << 24))) {
            if (p_bf16) g_bf16 ? launch_batch<uint16_t, uint16_t>(b, bits, stream) : launch_batch<uint16_t, float>(b, bits, stream);
            else g_bf16 ? launch_batch<float, uint16_t>(b, bits, stream) : launch_batch<float, float>(b, bits, stream);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            b.count = 0;
        }
    }
    return hipSuccess;
}

hipError_t launch_adamw_coef(double lr, double beta1, double beta2, double decay, const float *lr_dev, int32_t *step,
                             float *coef, hipStream_t stream) {
    hipLaunchKernelGGL(adamw_coef_kernel, dim3(1), dim3(1), 0, stream, lr, beta1, beta2, decay, lr_dev, step, coef);
    return hipGetLastError();
}

hipError_t launch_adamw_moments(const uint8_t *mc, const float *ms, const uint8_t *vc, const float *vs, int64_t n, float *m,
                                float *v, hipStream_t stream) {
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL(adamw_moments_kernel, dim3((unsigned)((n + kThreads * 4 - 1) / (kThreads * 4))), dim3(kThreads), 0, stream, mc,
                       ms, vc, vs, n, m, v);
    return hipGetLastError();
}

}  // namespace reqat
