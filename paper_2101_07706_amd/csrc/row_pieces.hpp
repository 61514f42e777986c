// Loads and stores of feature rows that start on any element: pieces of V values a lane, float or bfloat16 in memory, float in
// registers.
#pragma once
#include "common.hpp"

namespace csgs {

template <int V>
struct Vec {
    float x[V];
};

// Rows of the gathered tables are read through pointers that come out of LDS or a lane exchange as plain
// integers; the loads say that they go to global memory (a pointer of unknown kind would be read with the
// slower flat instructions, which every wait for LDS data would then wait for as well).
#define CSGS_GLOBAL __attribute__((address_space(1)))
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// A value in a table whose rows start on any element of ALIGN bytes: global loads and stores of any width take any address on this
// part, but the compiler has to know that they are asked to.  (A struct, whose alignment is part of the type: that of a typedef is
// dropped where it is a template argument, and the access then claims the vector's own.)
template <typename U, int ALIGN>
struct __attribute__((packed, aligned(ALIGN))) Piece {
    U v;
};
template <typename U, int ALIGN = (int)alignof(U)>
__device__ inline U load_global(const void *p)
{
    static_assert(alignof(Piece<U, ALIGN>) == ALIGN && sizeof(Piece<U, ALIGN>) == sizeof(U), "the claim on the address");
    return reinterpret_cast<const CSGS_GLOBAL Piece<U, ALIGN> *>((uintptr_t)p)->v;
}
template <typename U, int ALIGN = (int)alignof(U)>
__device__ inline void store_global(void *p, U v)
{
    static_assert(alignof(Piece<U, ALIGN>) == ALIGN && sizeof(Piece<U, ALIGN>) == sizeof(U), "the claim on the address");
    reinterpret_cast<CSGS_GLOBAL Piece<U, ALIGN> *>((uintptr_t)p)->v = v;
}

template <typename T, int V>
__device__ inline Vec<V> load_row(const T *p);

template <>
__device__ inline Vec<1> load_row<float, 1>(const float *p) { return Vec<1>{{load_global<float>(p)}}; }
template <>
__device__ inline Vec<2> load_row<float, 2>(const float *p)
{
    const f32x2 v = load_global<f32x2, 4>(p);
    return Vec<2>{{v.x, v.y}};
}
template <>
__device__ inline Vec<4> load_row<float, 4>(const float *p)
{
    const f32x4 v = load_global<f32x4, 4>(p);
    return Vec<4>{{v.x, v.y, v.z, v.w}};
}
template <>
__device__ inline Vec<8> load_row<float, 8>(const float *p)   // two 16-byte loads
{
    const f32x4 a = load_global<f32x4, 4>(p), b = load_global<f32x4, 4>(p + 4);
    return Vec<8>{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
// bfloat16 bit patterns: widening is a 16-bit left shift
template <>
__device__ inline Vec<1> load_row<uint16_t, 1>(const uint16_t *p) { return Vec<1>{{__uint_as_float((uint32_t)load_global<uint16_t>(p) << 16)}}; }
template <>
__device__ inline Vec<2> load_row<uint16_t, 2>(const uint16_t *p)
{
    const uint32_t v = load_global<uint32_t, 2>(p);
    return Vec<2>{{__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)}};
}
template <>
__device__ inline Vec<4> load_row<uint16_t, 4>(const uint16_t *p)
{
    const u32x2 v = load_global<u32x2, 2>(p);
    return Vec<4>{{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                   __uint_as_float(v.y & 0xFFFF0000u)}};
}
template <>
__device__ inline Vec<8> load_row<uint16_t, 8>(const uint16_t *p)
{
    const u32x4 v = load_global<u32x4, 2>(p);
    return Vec<8>{{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                   __uint_as_float(v.y & 0xFFFF0000u), __uint_as_float(v.z << 16), __uint_as_float(v.z & 0xFFFF0000u),
                   __uint_as_float(v.w << 16), __uint_as_float(v.w & 0xFFFF0000u)}};
}

// A piece as it lies in memory: what is asked for in one place and widened in another, so that many can be on their way (a value
// that is widened where it is loaded is waited for there, at the end of the branch at the latest).
template <typename T, int V>
struct RawPiece {
    static constexpr int WORDS = ((int)sizeof(T) * V + 3) / 4;
    static_assert(WORDS == 1 || WORDS == 2 || WORDS == 4 || WORDS == 8, "piece widths");
    uint32_t w[WORDS];   // (a single bfloat16: the lower half of one)
    __device__ void load(const T *p)
    {
        if constexpr (sizeof(T) * V == 2) w[0] = load_global<uint16_t>(p);
        else if constexpr (WORDS == 1) w[0] = load_global<uint32_t, (int)sizeof(T)>(p);
        if constexpr (WORDS == 2) {
            const u32x2 a = load_global<u32x2, (int)sizeof(T)>(p);
            w[0] = a.x; w[1] = a.y;
        }
        if constexpr (WORDS >= 4)
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) {
                const u32x4 a = load_global<u32x4, (int)sizeof(T)>((const uint32_t *)p + k);
                w[k] = a.x; w[k + 1] = a.y; w[k + 2] = a.z; w[k + 3] = a.w;
            }
    }
    __device__ float value(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
};

// The same the other way: a row's values to memory, bfloat16 by rounding to nearest even (NaN stays NaN).
__device__ inline uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x); }
// A double as the float that store_row is given for it, rounded once: for bfloat16 to one of its numbers, which store_row then keeps as it is.
template <typename T>
__device__ inline float float_to_store(double d)
{
    if constexpr (sizeof(T) == 4) return (float)d;
    return (float)(__bf16)d;
}
template <typename T, int V>
__device__ inline void store_row(T *p, const Vec<V> &v)
{
    static_assert(V == 1 || V == 2 || V == 4 || V == 8, "piece widths");
    if constexpr (sizeof(T) == 4) {
        if constexpr (V == 1) store_global<float>(p, v.x[0]);
        if constexpr (V == 2) store_global<f32x2, 4>(p, f32x2{v.x[0], v.x[1]});
        if constexpr (V == 4) store_global<f32x4, 4>(p, f32x4{v.x[0], v.x[1], v.x[2], v.x[3]});
        if constexpr (V == 8) {
            store_global<f32x4, 4>(p, f32x4{v.x[0], v.x[1], v.x[2], v.x[3]});
            store_global<f32x4, 4>(p + 4, f32x4{v.x[4], v.x[5], v.x[6], v.x[7]});
        }
    } else {
        auto two = [&](int i) { return bf16_bits(v.x[i]) | bf16_bits(v.x[i + 1]) << 16; };
        if constexpr (V == 1) store_global<uint16_t>(p, (uint16_t)bf16_bits(v.x[0]));
        if constexpr (V == 2) store_global<uint32_t, 2>(p, two(0));
        if constexpr (V == 4) store_global<u32x2, 2>(p, u32x2{two(0), two(2)});
        if constexpr (V == 8) store_global<u32x4, 2>(p, u32x4{two(0), two(2), two(4), two(6)});
    }
}
// 16 bytes past the caches, for what is too long to be found there again.
typedef u32x4 __attribute__((aligned(2))) u32x4_anywhere;
__device__ inline void store_past_caches(void *p, u32x4 v) { __builtin_nontemporal_store(v, (CSGS_GLOBAL u32x4_anywhere *)(uintptr_t)p); }
template <typename T, int V>
__device__ inline void store_row_past_caches(T *p, const Vec<V> &v)
{
    if constexpr (sizeof(T) * V != 16) store_row<T, V>(p, v);
    else if constexpr (sizeof(T) == 4)
        store_past_caches(p, u32x4{__float_as_uint(v.x[0]), __float_as_uint(v.x[1]), __float_as_uint(v.x[2]), __float_as_uint(v.x[3])});
    else {
        auto two = [&](int i) { return bf16_bits(v.x[i]) | bf16_bits(v.x[i + 1]) << 16; };
        store_past_caches(p, u32x4{two(0), two(2), two(4), two(6)});
    }
}
}  // namespace csgs
