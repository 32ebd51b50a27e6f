// Rows of float32, float16 or bfloat16 elements as 16-byte vectors, from any element-aligned address: gfx950 loads and
// stores 16 bytes at any alignment in one instruction, so rows of odd strides need no loads of their own - only other cache hints,
// where two rows share a line.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/sdtw.h"

namespace sdtw {

struct Bf16 { uint16_t bits; };

// 16 bytes as they lie in memory.  They stay packed until an element is used: unpacking right behind a load would wait for it.
typedef uint32_t Bits4 __attribute__((ext_vector_type(4)));
typedef Bits4 Bits4Any __attribute__((aligned(2)));

typedef float Float2 __attribute__((ext_vector_type(2)));

template <typename T> struct Elem;

template <> struct Elem<float> {
    static constexpr int kWidth = 4;  // elements of a 16-byte vector
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
    static __device__ __forceinline__ float at(const Bits4 &b, int e) { return __uint_as_float(b[e]); }
    static __device__ __forceinline__ Bits4 pack(const float (&x)[4])
    {
        return Bits4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
    static __device__ __forceinline__ void copy(Bits4 &b, int e, const Bits4 &from) { b[e] = from[e]; }
};
// one 16-bit element of a vector as it is
__device__ __forceinline__ void copy_half(Bits4 &b, int e, const Bits4 &from)
{
    const uint32_t mask = e & 1 ? 0xffff0000u : 0xffffu;
    b[e >> 1] = (b[e >> 1] & ~mask) | (from[e >> 1] & mask);
}

template <> struct Elem<_Float16> {
    static constexpr int kWidth = 8;
    typedef _Float16 Pair __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ float up(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 down(float v) { return (_Float16)v; }
    static __device__ __forceinline__ float at(const Bits4 &b, int e)
    {
        const uint32_t w = b[e >> 1];
        const uint16_t h = (uint16_t)(e & 1 ? w >> 16 : w);
        return (float)__builtin_bit_cast(_Float16, h);
    }
    static __device__ __forceinline__ uint32_t pack2(float lo, float hi)
    {
        const Float2 f = {lo, hi};
        const Pair p = __builtin_convertvector(f, Pair);
        return __builtin_bit_cast(uint32_t, p);
    }
    static __device__ __forceinline__ Bits4 pack(const float (&x)[8])
    {
        return Bits4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
    }
    static __device__ __forceinline__ void copy(Bits4 &b, int e, const Bits4 &from) { copy_half(b, e, from); }
};
template <> struct Elem<Bf16> {
    static constexpr int kWidth = 8;
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ float up(Bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
    static __device__ __forceinline__ Bf16 down(float v)
    {
        return Bf16{__builtin_bit_cast(uint16_t, (__bf16)v)};  // to nearest, ties to even; a NaN stays one
    }
    static __device__ __forceinline__ float at(const Bits4 &b, int e)
    {
        return __uint_as_float(e & 1 ? b[e >> 1] & 0xffff0000u : b[e >> 1] << 16);
    }
    static __device__ __forceinline__ uint32_t pack2(float lo, float hi)
    {
        const Float2 f = {lo, hi};
        const Pair p = __builtin_convertvector(f, Pair);
        return __builtin_bit_cast(uint32_t, p);
    }
    static __device__ __forceinline__ Bits4 pack(const float (&x)[8])
    {
        return Bits4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
    }
    static __device__ __forceinline__ void copy(Bits4 &b, int e, const Bits4 &from) { copy_half(b, e, from); }
};

// element e of a vector, as it is
template <typename T> __device__ __forceinline__ T element(const Bits4 &b, int e)
{
    const uint32_t v = b[sizeof(T) == 4 ? e : e >> 1];  // (a bit cast of b[e] itself is taken of element 0 by this compiler)
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, v);
    else return __builtin_bit_cast(T, (uint16_t)(e & 1 ? v >> 16 : v));
}

// STREAM: the non-temporal hint, for data that is used once.  Reading 4 GiB takes 7.1 TB/s with it and 6.2 without; copying
// 5.6 and 5.4 from and to whole cache lines, but 4.6 and 5.2 where rows start at odd 2-byte elements (half-written lines).
template <bool STREAM, typename T> __device__ __forceinline__ Bits4 load_vec(const T *p)
{
    const Bits4Any *q = reinterpret_cast<const Bits4Any *>(p);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
}

template <bool STREAM, typename T> __device__ __forceinline__ void store_vec(T *p, const Bits4 &b)
{
    Bits4Any *q = reinterpret_cast<Bits4Any *>(p);
    if (STREAM)
        __builtin_nontemporal_store(b, q);
    else
        *q = b;
}

// The vector moved down (shift > 0) or up by a number of bits below 128, zeros coming in.
__device__ __forceinline__ Bits4 shift_vec(const Bits4 &v, int shift)
{
    unsigned __int128 x = __builtin_bit_cast(unsigned __int128, v);
    x = shift >= 0 ? x >> shift : x << -shift;
    return __builtin_bit_cast(Bits4, x);
}

// The same at a byte offset from a row's start, for a row that all lanes share: its address goes into scalar registers, and the
// offset alone takes a vector register.
typedef __attribute__((address_space(1))) Bits4Any GlobalBits4;
typedef __attribute__((address_space(1))) char GlobalByte;
__device__ __forceinline__ GlobalByte *shared_row(const void *p)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return reinterpret_cast<GlobalByte *>((uint64_t)hi << 32 | lo);
}
template <bool STREAM> __device__ __forceinline__ Bits4 load_at(GlobalByte *row, uint32_t offset)
{
    GlobalBits4 *q = reinterpret_cast<GlobalBits4 *>(row + offset);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
}
template <bool STREAM> __device__ __forceinline__ void store_at(GlobalByte *row, uint32_t offset, const Bits4 &b)
{
    GlobalBits4 *q = reinterpret_cast<GlobalBits4 *>(row + offset);
    if (STREAM)
        __builtin_nontemporal_store(b, q);
    else
        *q = b;
}

// Element `i` of an array whose type is known at run time (SDTW_TYPE_*): for the few values of a row.
__device__ __forceinline__ float load_typed(const void *p, int64_t i, int type)
{
    if (type == SDTW_TYPE_F32) return static_cast<const float *>(p)[i];
    if (type == SDTW_TYPE_F16) return (float)static_cast<const _Float16 *>(p)[i];
    return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
}

// Sums and maxima over the 64 lanes of a wavefront, the same value in every lane.  Shifts within rows of 16 lanes, then lane 15
// of a row to the next one and lane 31 to the upper half: lane 63 holds the result (a lane without a partner gets the
// operation's neutral element).
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_f32(float v, float neutral)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(neutral), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_f64(double v)
{
    const long long b = __double_as_longlong(v);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double((long long)(((unsigned long long)(unsigned)hi << 32) | (unsigned)lo));
}
__device__ __forceinline__ float wave_sum_all_f32(float v)
{
    v += dpp_f32<0x111, 0xf>(v, 0.0f);
    v += dpp_f32<0x112, 0xf>(v, 0.0f);
    v += dpp_f32<0x114, 0xf>(v, 0.0f);
    v += dpp_f32<0x118, 0xf>(v, 0.0f);
    v += dpp_f32<0x142, 0xa>(v, 0.0f);
    v += dpp_f32<0x143, 0xc>(v, 0.0f);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max_all_f32(float v)
{
    v = fmaxf(v, dpp_f32<0x111, 0xf>(v, -INFINITY));
    v = fmaxf(v, dpp_f32<0x112, 0xf>(v, -INFINITY));
    v = fmaxf(v, dpp_f32<0x114, 0xf>(v, -INFINITY));
    v = fmaxf(v, dpp_f32<0x118, 0xf>(v, -INFINITY));
    v = fmaxf(v, dpp_f32<0x142, 0xa>(v, -INFINITY));
    v = fmaxf(v, dpp_f32<0x143, 0xc>(v, -INFINITY));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ double wave_sum_f64(double v)
{
    v += dpp_f64<0x111, 0xf>(v);
    v += dpp_f64<0x112, 0xf>(v);
    v += dpp_f64<0x114, 0xf>(v);
    v += dpp_f64<0x118, 0xf>(v);
    v += dpp_f64<0x142, 0xa>(v);
    v += dpp_f64<0x143, 0xc>(v);
    const long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)b, 63), hi = (unsigned)__builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
}

}  // namespace sdtw
