// Rows of bfloat16 or FP32 in 16-byte vectors, at any element alignment and of any length, and sums over a workgroup.
//
// A vector's address need only be aligned to its elements (gfx950 serves global accesses of 16 bytes at any address), so
// odd leading dimensions and odd lengths take the same path as even ones; only the last, partial vector of a row goes
// element by element.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace reqat {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Elements of a 16-byte vector: 8 bfloat16 (held as uint16_t) or 4 FP32.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) {   // to nearest, ties to even
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

template <typename T> __device__ __forceinline__ uint4 load_vec(const T *p) {
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T> __device__ __forceinline__ void store_vec(T *p, uint4 v) { __builtin_memcpy(p, &v, 16); }

// The same for data that a call touches once: it is not kept in the caches.
typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> __device__ __forceinline__ void store_vec_once(T *p, uint4 v) {
    __builtin_nontemporal_store(__builtin_bit_cast(Words, v), reinterpret_cast<Words *>(p));
}

// The first n elements of a vector (0 < n < kVec), zeros behind them.
template <typename T> __device__ __forceinline__ uint4 load_part(const T *p, int n) {
    T e[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) e[i] = i < n ? p[i] : T(0);
    return __builtin_bit_cast(uint4, e);
}
template <typename T> __device__ __forceinline__ void store_part(T *p, uint4 v, int n) {
    T e[kVec<T>];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
        if (i < n) p[i] = e[i];
}

template <typename T> __device__ __forceinline__ void unpack(uint4 v, float (&z)[kVec<T>]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[2 * i] = __uint_as_float(w[i] << 16);
            z[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <typename T> __device__ __forceinline__ uint4 pack(const float (&z)[kVec<T>]) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = (uint32_t)from_f32<uint16_t>(z[2 * i]) | ((uint32_t)from_f32<uint16_t>(z[2 * i + 1]) << 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sum over the 64 lanes, the same in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

}  // namespace reqat
