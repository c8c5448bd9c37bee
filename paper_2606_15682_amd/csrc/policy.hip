// Clipped policy loss with a KL term for gfx950, per token t (a row of logits z, p = softmax(z / temperature)):
//   lp = log p_y,  r = exp(lp - old),  x = ref - lp,
//   loss_t = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(x) - x - 1),   L = sum_t w_t loss_t,
//   dL/dlp = w_t (-A r [inside] - kl (exp(x) - 1)),  inside: neither A > 0, r > 1 + high nor A < 0, r < 1 - low,
//   dL/dz_j = (dL/dlp) ([j = y] - p_j) / temperature.
//
// Softmax statistics relative to the largest logit m: terms 2^t, t = (z - m) c, c = log2(e) / temperature, S their sum.  The
// difference comes first: it is exact for the likely tokens, whose 1 - p is small, costs no digits where all logits are large,
// and keeps its meaning up to the type's largest and lowest values, where c z is past FP32's range.
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

constexpr int kThreads = 512;
constexpr int kMaxHeld = 18;

// The base-2 exponent of a difference d <= 0, which may be -Inf.  FP32 rows take what the factor's rounding leaves too: that
// error is the same in every term, c_rest / c of the distance to the maximum, where the other roundings average out.
template <typename T> __device__ __forceinline__ float exponent(const PolicyArgs &a, float d) {
    return sizeof(T) == 4 ? __builtin_fmaf(d, a.c, d * a.c_rest) : d * a.c;
}

// Running maximum and sum of a slice of a row; empty, and so for a slice of -Inf logits alone: m = -Inf, S = 0.
struct Online {
    float m, S;
};

// What exponents are relative to: the maximum, or a number that leaves -Inf what it is.
__device__ __forceinline__ float reference(float m) { return __builtin_fmaxf(m, -3.402823466e38f); }

// A NaN logit makes S NaN, and so does +Inf (Inf - Inf): the row's statistics are NaN then.
template <typename T> __device__ __forceinline__ void add(Online &o, const PolicyArgs &a, uint4 v) {
    constexpr int N = kVec<T>;
    float z[N];
    unpack<T>(v, z);
    float mx = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) mx = __builtin_fmaxf(mx, z[i]);
    if (mx > o.m) {
        if (o.S != 0.0f) o.S *= __builtin_amdgcn_exp2f(exponent<T>(a, o.m - mx));
        o.m = mx;
    }
    const float ref = reference(o.m);
    float sum = 0.0f;                       // of the vector first: single small terms would be lost beside a large S
#pragma unroll
    for (int i = 0; i < N; ++i) sum += __builtin_amdgcn_exp2f(exponent<T>(a, z[i] - ref));
    o.S += sum;
}

template <typename T> __device__ __forceinline__ Online merge(const PolicyArgs &args, Online a, Online b) {
    if (b.m > a.m) { const Online t = a; a = b; b = t; }
    if (b.S == 0.0f) return a;
    a.S += b.S * __builtin_amdgcn_exp2f(exponent<T>(args, b.m - a.m));
    return a;
}

// The workgroup's TH slices in a fixed order: within the wave, then wave by wave.
template <typename T, int TH> __device__ __forceinline__ Online join(const PolicyArgs &a, Online o, Online (&red)[TH / 64]) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) o = merge<T>(a, o, Online{__shfl_xor(o.m, off, 64), __shfl_xor(o.S, off, 64)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = o;
    __syncthreads();
    o = red[0];
#pragma unroll
    for (int k = 1; k < TH / 64; ++k) o = merge<T>(a, o, red[k]);
    return o;
}

// exp(x) - x - 1 >= 0.  Near zero the difference of close numbers is summed as its series (to x^8 / 8!: 5e-8 of it at 1/2).
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

// What a row brings besides its logits, asked for before they are summed.
struct RowInputs {
    float w, old, adv, ref, zy;
    int32_t y;
};

// A number at an address that is the same in every lane, read through the scalar cache: no vector register, and no wait for
// the vector loads in flight.  Nothing that this kernel writes is read so.
template <typename T> __device__ __forceinline__ T load_scalar(const T *p) {
    static_assert(sizeof(T) == 4, "a word");
    return *(const __attribute__((address_space(4))) T *)reinterpret_cast<uintptr_t>(p);
}

// An element of a row, by the word that holds it.
__device__ __forceinline__ float scalar_element(const float *p) { return load_scalar(p); }
__device__ __forceinline__ float scalar_element(const uint16_t *p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint32_t w = load_scalar(reinterpret_cast<const uint32_t *>(at & ~(uintptr_t)3));
    return __uint_as_float(at & 2 ? w & 0xFFFF0000u : w << 16);
}

__device__ __forceinline__ float weight_of(const PolicyArgs &a, int64_t t) {
    return a.weights ? load_scalar(a.weights + t) : a.default_weight;
}

// A number that is the same in every lane, in a scalar register.
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// All but the target's logit.
__device__ __forceinline__ RowInputs row_inputs(const PolicyArgs &a, int64_t t) {
    RowInputs in;
    in.zy = __builtin_nanf("");
    in.y = load_scalar(a.targets + t);
    in.w = weight_of(a, t);
    in.old = load_scalar(a.old_logp + t);
    in.adv = load_scalar(a.adv + t);
    in.ref = a.ref ? load_scalar(a.ref + t) : 0.0f;
    return in;
}

// A target outside [0, V) gives a NaN logit; what is read for it is the row's first one.  (With grad in the logits' memory
// this is still before the row is written, by this workgroup.)
template <typename T> __device__ __forceinline__ RowInputs row_inputs(const PolicyArgs &a, int64_t t, const T *row) {
    RowInputs in = row_inputs(a, t);
    const bool known = in.y >= 0 && (int64_t)in.y < a.V;
    const float zy = scalar_element(row + (known ? in.y : 0));
    if (known) in.zy = zy;
    return in;
}

// lp, log-sum-exp, dL/dlp and r of a row.
__device__ __forceinline__ float4 row_stats(const PolicyArgs &a, const RowInputs &in, Online o) {
    const float ref = reference(o.m), lnS = __builtin_amdgcn_logf(o.S) * kLn2;
    const float lp = (in.zy - ref) / a.temp - lnS, lse = ref / a.temp + lnS;
    const float r = expf(lp - in.old);
    float slope = outside(a, r, in.adv) ? 0.0f : -in.adv * r;
    if (a.ref && a.kl != 0.0f) slope -= a.kl * expm1f(in.ref - lp);      // not 0 times Inf
    return make_float4(lp, lse, in.w * slope, r);
}

// dL/dz of a vector whose first element is j: f [j = y] - fs 2^t.
template <typename T>
__device__ __forceinline__ uint4 grad_vec(const PolicyArgs &a, uint4 v, float ref, float fs, float f, int32_t j, int32_t y) {
    constexpr int N = kVec<T>;
    float z[N];
    unpack<T>(v, z);
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = -fs * __builtin_amdgcn_exp2f(exponent<T>(a, z[i] - ref));
    if ((uint32_t)(y - j) < (uint32_t)N) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] += j + i == y ? f : 0.0f;
    }
    return pack<T>(z);
}

// Vector j of a row of V elements; -Inf, whose exponential is 0, behind its end.
template <typename T> __device__ __forceinline__ uint4 load_at(const T *row, int32_t V, int32_t j) {
    constexpr int N = kVec<T>;
    if (V - j >= N) return load_vec(row + j);
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = j + i < V ? row[j + i] : from_f32<T>(-__builtin_inff());
    return __builtin_bit_cast(uint4, e);
}

template <typename T> __device__ __forceinline__ void store_at(T *row, int32_t V, int32_t j, uint4 v) {
    if (V - j >= kVec<T>) store_vec(row + j, v);
    else store_part(row + j, v, V - j);
}

// The gradient of the elements [begin, end) of a row (begin a multiple of the vector), by TH threads.
template <typename T, int TH>
__device__ __forceinline__ void write_grad(const PolicyArgs &a, const T *row, T *out, int32_t begin, int32_t end, float ref,
                                           float fs, float f, int32_t y) {
    for (int32_t j = begin + (int32_t)threadIdx.x * kVec<T>; j < end; j += TH * kVec<T>)
        store_at(out, end, j, grad_vec<T>(a, load_at(row, end, j), ref, fs, f, j, y));
}

template <typename T, int TH> __device__ __forceinline__ void write_zeros(T *out, int32_t begin, int32_t end) {
    for (int32_t j = begin + (int32_t)threadIdx.x * kVec<T>; j < end; j += TH * kVec<T>) store_at(out, end, j, make_uint4(0, 0, 0, 0));
}

// Loss alone: a workgroup per row, which is read once.
template <typename T> __global__ __launch_bounds__(kThreads) void policy_rows_kernel(PolicyArgs a) {
    constexpr int N = kVec<T>, kStep = kThreads * N;
    const int64_t t = blockIdx.x;
    const float w = weight_of(a, t);
    if (w == 0.0f) {
        if (threadIdx.x == 0) reinterpret_cast<float4 *>(a.stats)[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        return;
    }
    const T *row = reinterpret_cast<const T *>(a.logits) + t * a.ld;
    const RowInputs in = row_inputs(a, t, row);
    Online o{-__builtin_inff(), 0.0f};
    const int64_t V = a.V;
    int64_t j = (int64_t)threadIdx.x * N;
    for (; j + 3 * kStep + N <= V; j += 4 * kStep) {
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = load_vec(row + j + u * kStep);
#pragma unroll
        for (int u = 0; u < 4; ++u) add<T>(o, a, v[u]);
    }
    for (; j < V; j += kStep) add<T>(o, a, load_at(row, (int32_t)V, (int32_t)j));
    __shared__ Online red[kThreads / 64];
    o = join<T, kThreads>(a, o, red);
    if (threadIdx.x == 0) reinterpret_cast<float4 *>(a.stats)[t] = row_stats(a, in, o);
}

// Vector v as it came, after x is known: without this the compiler unpacks all vectors of a row first, or keeps the unpacked
// ones from the sums to the gradients, in two or four times the registers.
__device__ __forceinline__ void pin(uint4 &v, float x) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w) : "v"(x)); }

// Loss and gradient.  Workgroups of TH threads walk over the rows in steps of the grid and keep a row's first TH x NV
// whole vectors in registers, so that most rows are read once; as the gradient of a vector is written, the next row's is
// asked for in its place.  What does not fit, and a last partial vector, is read again, from the caches.  logits and grad
// may be the same memory: a row's vectors are read before they are written, and the next row is another one's memory.
//
// The row has more than (NV - 1) TH whole vectors (or NV is 0), so that all but the last step's accesses are without a
// condition: behind a branch the compiler cannot count the accesses in flight, and waits for all of them.
//
// 4096 rows of 152064 bfloat16 logits, a quarter without weight, take 474 us, 4.6 TB/s of one read and one write (a large
// copy: 5.2); with 17 of its 19 vectors a thread held and the others read again 9 us more, with 15 35 us more.  All 19 take
// three registers more than there are (12 bytes of scratch) and 2 us less; rows of 18 vectors are 2 us slower then.  A form that
// read every row twice, the second time from the caches, took 615 us.
template <typename T, int TH, int NV> __global__ __launch_bounds__(TH) void policy_grad_kernel(PolicyArgs a) {
    constexpr int N = kVec<T>, kStep = TH * N, kHeld = kStep * NV, kBytes = TH * 16;
    const int32_t V = (int32_t)a.V, j0 = threadIdx.x * N, full = V / N * N, rest = full < kHeld ? full : kHeld;
    const uint32_t lane = threadIdx.x * 16;             // bytes from a step's begin, which is the same in every lane
    const bool last = j0 < full - (NV - 1) * kStep;     // whether the last step has a vector of this thread
    const T *logits = reinterpret_cast<const T *>(a.logits);
    T *grad = reinterpret_cast<T *>(a.grad);
    __shared__ Online red[2][TH / 64];
    int half = 0;
    uint4 buf[NV > 0 ? NV : 1];
    // the next row with a weight from t on; those without get their zeros
    const auto seek = [&](int64_t t) {
        for (; t < a.T; t += gridDim.x) {
            if (weight_of(a, t) != 0.0f) break;
            if (threadIdx.x == 0) reinterpret_cast<float4 *>(a.stats)[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            write_zeros<T, TH>(grad + t * a.ldg, 0, V);
        }
        return t;
    };
    int64_t t = seek(blockIdx.x);
    if (t >= a.T) return;
    const T *row = logits + t * a.ld;
    RowInputs in = row_inputs(a, t, row);
#pragma unroll
    for (int v = 0; v < NV; ++v)
        if (v < NV - 1 || last) buf[v] = load_vec(reinterpret_cast<const char *>(row) + v * kBytes + lane);
    while (true) {
        const int32_t y = in.y;
        Online o{-__builtin_inff(), 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            pin(buf[v], o.S);
            if (v < NV - 1 || last) add<T>(o, a, buf[v]);
        }
        for (int32_t j = j0 + rest; j < V; j += kStep) add<T>(o, a, load_at(row, V, j));
        o = join<T, TH>(a, o, red[half]);
        half ^= 1;                                      // the other half is written before this one is again
        const float ref = uniform(reference(o.m));
        const float4 s = row_stats(a, in, o);
        if (threadIdx.x == 0) reinterpret_cast<float4 *>(a.stats)[t] = s;
        const float f = uniform(s.z / a.temp), fs = uniform(f / o.S);
        T *out = grad + t * a.ldg;
        const int64_t next = seek(t + gridDim.x);
        const bool more = next < a.T;
        // no further row: this one's first vector once more, for all steps
        const T *ahead = logits + (more ? next : t) * a.ld;
        const uint32_t hop = more ? kBytes : 0;
        in = row_inputs(a, more ? next : t, ahead);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            pin(buf[v], ref);
            if (v < NV - 1 || last) {
                store_vec_once(reinterpret_cast<char *>(out) + v * kBytes + lane, grad_vec<T>(a, buf[v], ref, fs, f, j0 + v * kStep, y));
                buf[v] = load_vec(reinterpret_cast<const char *>(ahead) + v * hop + lane);
            }
        }
        write_grad<T, TH>(a, row, out, rest, V, ref, fs, f, y);
        if (!more) return;
        t = next;
        row = ahead;
    }
}

// The gradient from the statistics: a workgroup per row and slice of it.  p_j = 2^((z_j - z_y) c + lp log2(e)) or 2^(z_j c -
// lse log2(e)), by the smaller of |lp| and |lse|, whose rounding is the exponent's error; dL/dz_y = -f (exp(lp) - 1).
// 4096 x 152064 bfloat16 493 us, 5.05 TB/s, 64 rows 7.8 us; FP32 1024 rows 266 us, 4.7 TB/s.
// hold: z_y has to stay for the row's other workgroups, where grad takes the logits' place; a launch of its own follows.
template <typename T> __global__ __launch_bounds__(kThreads) void policy_backward_kernel(PolicyArgs a, int64_t slice, bool hold) {
    constexpr int N = kVec<T>;
    const int64_t t = blockIdx.x;
    const int32_t begin = (int32_t)(blockIdx.y * slice), end = (int32_t)(begin + slice < a.V ? begin + slice : a.V);
    const T *row = reinterpret_cast<const T *>(a.logits) + t * a.ld;
    T *out = reinterpret_cast<T *>(a.grad) + t * a.ldg;
    const float4 s = reinterpret_cast<const float4 *>(a.stats)[t];
    if (s.z == 0.0f) {                                     // no weight, or clipped without a KL term: nothing to read
        write_zeros<T, kThreads>(out, begin, end);
        return;
    }
    const int32_t y = a.targets[t];
    const float f = s.z / a.temp * (a.grad_loss ? a.grad_loss[0] : 1.0f), fy = -f * expm1f(s.x);
    const bool by_target = __builtin_fabsf(s.x) < __builtin_fabsf(s.y) && y >= 0 && y < a.V;
    const float base = by_target ? to_f32(row[y]) : 0.0f, shift = (by_target ? s.x : -s.y) * kLog2e;
    if (!hold) __syncthreads();                            // all have read z_y
    for (int32_t j = begin + (int32_t)threadIdx.x * N; j < end; j += kThreads * N) {
        float z[N];
        unpack<T>(load_at(row, end, j), z);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = z[i] - base;
            z[i] = -f * __builtin_amdgcn_exp2f(__builtin_fmaf(d, a.c, sizeof(T) == 4 ? __builtin_fmaf(d, a.c_rest, shift) : shift));
        }
        const bool here = (uint32_t)(y - j) < (uint32_t)N;
        if (here) {
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = j + i == y ? fy : z[i];
        }
        if (here && hold) {
            T e[N];
            const uint4 v = pack<T>(z);
            __builtin_memcpy(e, &v, 16);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (j + i < end && j + i != y) out[j + i] = e[i];
        } else {
            store_at(out, end, j, pack<T>(z));
        }
    }
}

// The targets' elements, a thread each, where the rows were held.
template <typename T> __global__ __launch_bounds__(kThreads) void policy_backward_targets_kernel(PolicyArgs a) {
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (t >= a.T) return;
    const float4 s = reinterpret_cast<const float4 *>(a.stats)[t];
    const int32_t y = a.targets[t];
    if (s.z == 0.0f || y < 0 || y >= a.V) return;
    const float f = s.z / a.temp * (a.grad_loss ? a.grad_loss[0] : 1.0f);
    reinterpret_cast<T *>(a.grad)[t * a.ldg + y] = from_f32<T>(-f * expm1f(s.x));
}

constexpr int kSumThreads = 1024;

// Adds w surrogate, w KL and w [outside] of a row.
__device__ __forceinline__ void add_terms(const PolicyArgs &a, float w, float adv, float ref, float lp, float r, double (&s)[3]) {
    const float held = r < a.low ? a.low : (r > a.high ? a.high : r);
    const float x = r * adv, y = held * adv;
    s[0] += (double)w * -(double)(y < x ? y : x);
    if (a.ref) s[1] += (double)w * (double)kl_term(ref - lp);
    s[2] += outside(a, r, adv) ? (double)w : 0.0;
}

// loss = sum w (surrogate + kl KL), sum w surrogate, sum w KL, sum w [outside]; FP64, the threads' sums in a fixed order.
template <int TH> __device__ __forceinline__ void write_loss(const PolicyArgs &a, double (&s)[3]) {
    __shared__ double red[3][TH / 64];
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
            for (int i = 0; i < TH / 64; ++i) s[k] += red[k][i];
        }
        a.loss[0] = (float)(a.kl != 0.0f ? s[0] + (double)a.kl * s[1] : s[0]);
        a.loss[1] = (float)s[0];
        a.loss[2] = (float)s[1];
        a.loss[3] = (float)s[2];
    }
}

__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(PolicyArgs a) {
    double s[3] = {0.0, 0.0, 0.0};
    for (int64_t t = threadIdx.x; t < a.T; t += kSumThreads) {
        const float w = a.weights ? a.weights[t] : a.default_weight;
        if (w == 0.0f) continue;
        const float4 st = reinterpret_cast<const float4 *>(a.stats)[t];
        add_terms(a, w, a.adv[t], a.ref ? a.ref[t] : 0.0f, st.x, st.w, s);
    }
    write_loss<kSumThreads>(a, s);
}

// ------------------------------------------------------------------ few rows: several workgroups to a row

// Statistics of slice blockIdx.y of row blockIdx.x, and the target's logit where it is in the slice: the gradient may be
// written over the logits by then.
template <typename T> __global__ __launch_bounds__(kThreads) void policy_part_kernel(PolicyArgs a, int32_t slice) {
    const int64_t t = blockIdx.x;
    if (weight_of(a, t) == 0.0f) return;
    const int32_t V = (int32_t)a.V, begin = (int32_t)blockIdx.y * slice, end = V - begin < slice ? V : begin + slice;
    const T *row = reinterpret_cast<const T *>(a.logits) + t * a.ld;
    Online o{-__builtin_inff(), 0.0f};
#pragma unroll 4
    for (int32_t j = begin + (int32_t)threadIdx.x * kVec<T>; j < end; j += kThreads * kVec<T>) add<T>(o, a, load_at(row, end, j));
    __shared__ Online red[kThreads / 64];
    o = join<T, kThreads>(a, o, red);
    if (threadIdx.x == 0) {
        const int32_t y = a.targets[t];
        a.parts[t * gridDim.y + blockIdx.y] = make_float4(o.m, o.S, y >= begin && y < end ? to_f32(row[y]) : __builtin_nanf(""), 0.0f);
    }
}

// A row's slices in their order, and its target's logit.
template <typename T>
__device__ __forceinline__ Online merge_parts(const PolicyArgs &a, int64_t t, int32_t slice, int slices, RowInputs &in) {
    Online o{-__builtin_inff(), 0.0f};
    for (int k = 0; k < slices; ++k) {
        const float4 p = a.parts[t * slices + k];
        o = merge<T>(a, o, Online{p.x, p.y});
        if (in.y >= 0 && in.y / slice == k) in.zy = p.z;      // NaN for a target behind the row's end
    }
    return o;
}

// Workgroup 0: every row's statistics, a thread each, and the loss.  Workgroup 1 + t slices + k: the gradient of slice k of
// row t.
template <typename T> __global__ __launch_bounds__(kThreads) void policy_finish_kernel(PolicyArgs a, int32_t slice, int slices) {
    if (blockIdx.x == 0) {
        double s[3] = {0.0, 0.0, 0.0};
        for (int64_t t = threadIdx.x; t < a.T; t += kThreads) {
            const float w = a.weights ? a.weights[t] : a.default_weight;
            float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (w != 0.0f) {
                RowInputs in = {w, a.old_logp[t], a.adv[t], a.ref ? a.ref[t] : 0.0f, __builtin_nanf(""), a.targets[t]};
                const Online o = merge_parts<T>(a, t, slice, slices, in);
                st = row_stats(a, in, o);
                add_terms(a, w, in.adv, in.ref, st.x, st.w, s);
            }
            reinterpret_cast<float4 *>(a.stats)[t] = st;
        }
        write_loss<kThreads>(a, s);
        return;
    }
    const int64_t t = (blockIdx.x - 1) / slices;
    const int32_t V = (int32_t)a.V, begin = (int32_t)((blockIdx.x - 1) % slices) * slice, end = V - begin < slice ? V : begin + slice;
    const T *row = reinterpret_cast<const T *>(a.logits) + t * a.ld;
    T *out = reinterpret_cast<T *>(a.grad) + t * a.ldg;
    if (weight_of(a, t) == 0.0f) {
        write_zeros<T, kThreads>(out, begin, end);
        return;
    }
    RowInputs in = row_inputs(a, t);
    const Online o = merge_parts<T>(a, t, slice, slices, in);
    const float f = row_stats(a, in, o).z / a.temp;
    write_grad<T, kThreads>(a, row, out, begin, end, reference(o.m), f / o.S, f, in.y);
}

}  // namespace

namespace {

// Workgroups of 256 threads for rows of up to 4096 bytes a wave, else of 1024, with as many vectors as the row has and the
// registers hold (128 a thread, with 18).  They are persistent: as many as the card's 256 compute units hold at once.
template <typename T, int TH, int NV> void launch_grad_of(const PolicyArgs &a, int64_t steps, hipStream_t stream) {
    if (steps == NV) {
        const int64_t most = TH == 256 ? 4 * 256 : 256;
        hipLaunchKernelGGL((policy_grad_kernel<T, TH, NV>), dim3((unsigned)(a.T < most ? a.T : most)), dim3(TH), 0, stream, a);
    } else if constexpr (NV > (TH == 256 ? 0 : 2)) {       // more than 1024 vectors are at least two of 1024 threads
        launch_grad_of<T, TH, NV - 1>(a, steps, stream);
    }
}

template <typename T> void launch_grad(const PolicyArgs &a, hipStream_t stream) {
    const int64_t full = a.V / kVec<T>, steps = (full + 1023) / 1024;
    if (full <= 4 * 256) launch_grad_of<T, 256, 4>(a, (full + 255) / 256, stream);
    else launch_grad_of<T, 1024, kMaxHeld>(a, steps < kMaxHeld ? steps : kMaxHeld, stream);
}

}  // namespace

hipError_t launch_policy_loss(const PolicyArgs &a, bool bf16, hipStream_t stream) {
    const dim3 grid((unsigned)a.T), block(kThreads);
    const PolicyPlan plan = policy_plan(a.T, a.V, bf16);
    if (plan.slices > 1) {
        const int32_t slice = (int32_t)plan.slice;
        const int slices = (int)plan.slices;
        const dim3 parts((unsigned)a.T, (unsigned)slices), finish(a.grad ? (unsigned)(1 + a.T * slices) : 1);
        if (bf16) {
            hipLaunchKernelGGL(policy_part_kernel<uint16_t>, parts, block, 0, stream, a, slice);
            hipLaunchKernelGGL(policy_finish_kernel<uint16_t>, finish, block, 0, stream, a, slice, slices);
        } else {
            hipLaunchKernelGGL(policy_part_kernel<float>, parts, block, 0, stream, a, slice);
            hipLaunchKernelGGL(policy_finish_kernel<float>, finish, block, 0, stream, a, slice, slices);
        }
        return hipGetLastError();
    }
    if (a.T > 0) {
        if (a.grad) bf16 ? launch_grad<uint16_t>(a, stream) : launch_grad<float>(a, stream);
        else if (bf16) hipLaunchKernelGGL(policy_rows_kernel<uint16_t>, grid, block, 0, stream, a);
        else hipLaunchKernelGGL(policy_rows_kernel<float>, grid, block, 0, stream, a);
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
    const int64_t cuts = (a.V + slice - 1) / slice;
    const bool hold = cuts > 1 && a.grad == a.logits;
    const dim3 grid((unsigned)a.T, (unsigned)cuts), block(kThreads), targets((unsigned)((a.T + kThreads - 1) / kThreads));
    if (bf16) hipLaunchKernelGGL(policy_backward_kernel<uint16_t>, grid, block, 0, stream, a, slice, hold);
    else hipLaunchKernelGGL(policy_backward_kernel<float>, grid, block, 0, stream, a, slice, hold);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !hold) return e;
    if (bf16) hipLaunchKernelGGL(policy_backward_targets_kernel<uint16_t>, targets, block, 0, stream, a);
    else hipLaunchKernelGGL(policy_backward_targets_kernel<float>, targets, block, 0, stream, a);
    return hipGetLastError();
}

}  // namespace reqat
