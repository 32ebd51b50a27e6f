// Rows of float32, float16 or bfloat16 elements as 16-byte vectors, from any element-aligned address: gfx950 loads and
// stores 16 bytes at any alignment in one instruction, so rows of odd strides need no path of their own.
#pragma once
#include <hip/hip_runtime.h>

#include <cstring>

#include "../../include/sdtw.h"

namespace sdtw {

struct Bf16 { uint16_t bits; };

template <typename T> struct Elem;

template <> struct Elem<float> {
    static constexpr int kWidth = 4;  // elements of a 16-byte vector
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <> struct Elem<_Float16> {
    static constexpr int kWidth = 8;
    static __device__ __forceinline__ float up(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 down(float v) { return (_Float16)v; }
};
template <> struct Elem<Bf16> {
    static constexpr int kWidth = 8;
    static __device__ __forceinline__ float up(Bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
    static __device__ __forceinline__ Bf16 down(float v)
    {
        const __bf16 r = (__bf16)v;  // to nearest, ties to even; a NaN stays one
        Bf16 o;
        __builtin_memcpy(&o, &r, 2);
        return o;
    }
};

template <typename T> struct Vec {
    static constexpr int W = Elem<T>::kWidth;
    T e[W];
};

template <typename T> __device__ __forceinline__ Vec<T> load_vec(const T *p)
{
    Vec<T> v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <typename T> __device__ __forceinline__ void store_vec(T *p, const Vec<T> &v) { __builtin_memcpy(p, &v, 16); }

// Element `i` of an array whose type is known at run time (SDTW_TYPE_*): for the few values of a row.
__device__ __forceinline__ float load_typed(const void *p, int64_t i, int type)
{
    if (type == SDTW_TYPE_F32) return static_cast<const float *>(p)[i];
    if (type == SDTW_TYPE_F16) return (float)static_cast<const _Float16 *>(p)[i];
    return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
}

// Sum and maximum over the 64 lanes, the same value in every lane.
__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}
__device__ __forceinline__ float wave_sum_all_f32(float v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}
__device__ __forceinline__ float wave_max_all_f32(float v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}

}  // namespace sdtw
