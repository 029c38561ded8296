// Rows of real values in 32 or 16 bits, read and written eight neighbours at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "xnor_lowbit.h"

namespace xnor {

template <int TYPE> struct RealType;
template <> struct RealType<XNOR_F32> { typedef float type; };
template <> struct RealType<XNOR_BF16> { typedef __bf16 type; };
template <> struct RealType<XNOR_F16> { typedef _Float16 type; };
template <int TYPE> using real_t = typename RealType<TYPE>::type;

// f(type as a constant) for one of the three types
template <class F> void by_type(int type, F f)
{
    if (type == XNOR_F32) f(std::integral_constant<int, XNOR_F32>());
    else if (type == XNOR_BF16) f(std::integral_constant<int, XNOR_BF16>());
    else f(std::integral_constant<int, XNOR_F16>());
}
inline bool known_type(int type) { return type == XNOR_F32 || type == XNOR_BF16 || type == XNOR_F16; }
inline size_t type_bytes(int type) { return type == XNOR_F32 ? 4 : 2; }

// 16 bytes that lie at any multiple of an element: rows of odd widths start there (the memory takes such accesses whole)
typedef uint32_t words4_any __attribute__((ext_vector_type(4), aligned(2)));

// Eight neighbouring values as they are stored, four to eight registers.
template <int TYPE> struct Real8 {
    typedef real_t<TYPE> T;
    static constexpr int QUADS = sizeof(T) * 8 / 16;
    union {
        words4_any quad[QUADS];
        T v[8];
    };
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
    // n: how many of the eight exist (more than eight: all); the others are `fill`
    __device__ __forceinline__ void load(const T *p, int n, float fill = 0.0f)
    {
        if (n >= 8) {
#pragma unroll
            for (int q = 0; q < QUADS; ++q) quad[q] = reinterpret_cast<const words4_any *>(p)[q];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)fill;
        }
    }
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if (n >= 8) {
#pragma unroll
            for (int q = 0; q < QUADS; ++q) reinterpret_cast<words4_any *>(p)[q] = quad[q];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = v[i];
        }
    }
};

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s, 64);
    return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, s, 64));
    return v;
}

}  // namespace xnor
