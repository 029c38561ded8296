// Rows and codes as operands of the matrix instructions: shared by the kernels of w4_linear.hip and w4_tiles.hip.
#pragma once
#include "real8.h"

namespace xnor {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// How rows meet the codes in the matrix instructions (16 x 16 x 32).  For 16-bit rows a code u enters as 16 + u, which two instructions per
// pair form: the top of the mantissa under a fixed exponent.  What that and the zero point add to a sum is the same multiple of the group's sum
// of x for all inputs and is taken out with it:
//     sum x (u - z) = sum x (16 + u) - (16 + z) sum x
// bfloat16 takes a 4096th of that, and the results are multiplied by it at the end: the sums of 128 inputs of float32's whole range stay within it.
// For 8-bit rows it enters as u - z, seven instructions for eight codes, and the sums are exact.  Float32 rows are three bfloat16 numbers each
// whose sum they are.
enum { ROWS_F32 = XNOR_F32, ROWS_BF16 = XNOR_BF16, ROWS_F16 = XNOR_F16, ROWS_I8 = 3 };

template <int X> struct Form {          // 16 bits
    static constexpr int PARTS = X == ROWS_F32 ? 3 : 1;
    static constexpr float OFFSET = 16.0f, BACK = X == ROWS_F16 ? 1.0f : 4096.0f;        // BACK: what a result is multiplied by
    typedef f32x4 acc_t;
    typedef u32x4 operand_t;
    static __device__ __forceinline__ operand_t ones()          // 1 / BACK
    {
        const uint32_t one = X == ROWS_F16 ? 0x3c003c00u : 0x39803980u;
        return operand_t{one, one, one, one};
    }
    static __device__ __forceinline__ operand_t widen(uint32_t w)
    {
        uint32_t mask = X == ROWS_F16 ? 0x03c003c0u : 0x00780078u, base = X == ROWS_F16 ? 0x4c004c00u : 0x3b803b80u;
        asm("" : "+v"(mask), "+v"(base));           // (in registers: an and-or takes no two literals)
        if (X == ROWS_F16) return operand_t{(w << 6 & mask) | base, (w << 2 & mask) | base, (w >> 2 & mask) | base, (w >> 6 & mask) | base};
        return operand_t{(w << 3 & mask) | base, (w >> 1 & mask) | base, (w >> 5 & mask) | base, (w >> 9 & mask) | base};
    }
    static __device__ __forceinline__ acc_t mfma(operand_t a, operand_t b, acc_t c)
    {
        if (X == ROWS_F16)
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Form<ROWS_I8> {
    static constexpr int PARTS = 1;
    typedef i32x4 acc_t;
    typedef long operand_t;             // bytes 0 4 1 5 2 6 3 7 of eight neighbours
    // z: the zero point in every byte
    static __device__ __forceinline__ uint32_t minus(uint32_t u, uint32_t z)
    {
        uint32_t mask = 0x0f0f0f0fu, top = 0x80808080u;
        asm("" : "+v"(mask), "+v"(top));
        return ((u & mask) | top) - z ^ top;
    }
    static __device__ __forceinline__ operand_t widen(uint32_t w, uint32_t z)
    {
        return (operand_t)((uint64_t)minus(w, z) | (uint64_t)minus(w >> 4, z) << 32);
    }
    static __device__ __forceinline__ acc_t mfma(operand_t a, operand_t b, acc_t c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0); }
};

// Eight neighbours of a row as operands (PARTS of them); n: how many exist, the others are 0.
template <int X> struct Eight;
template <int X> struct Eight {
    Real8<X> v;
    __device__ __forceinline__ void load(const void *row, int k, int n) { v.load(static_cast<const real_t<X> *>(row) + k, n); }
    __device__ __forceinline__ void operands(typename Form<X>::operand_t *b) const
    {
        if constexpr (X != ROWS_F32) {
            b[0] = v.quad[0];
        } else {
            // truncated to 8 bits of mantissa, then the rest, and the rest of that: exact (an infinity has no rest, a NaN stays one)
            uint32_t w[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t part[2][3];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float x = v[2 * i + h];
                    const bool finite = __builtin_fabsf(x) < __builtin_inff();
                    const uint32_t hi = (__float_as_uint(x) | (x != x ? 0x00400000u : 0u)) & 0xffff0000u;
                    const float rest = finite ? x - __uint_as_float(hi) : 0.0f;
                    const uint32_t mid = __float_as_uint(rest) & 0xffff0000u;
                    part[h][0] = hi;
                    part[h][1] = mid;
                    part[h][2] = __float_as_uint(rest - __uint_as_float(mid));
                }
#pragma unroll
                for (int p = 0; p < 3; ++p) w[p][i] = part[0][p] >> 16 | (part[1][p] & 0xffff0000u);
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) b[p] = u32x4{w[p][0], w[p][1], w[p][2], w[p][3]};
        }
    }
};
template <> struct Eight<ROWS_I8> {
    uint32_t w[2];
    __device__ __forceinline__ void load(const void *row, int k, int n)
    {
        const int8_t *p = static_cast<const int8_t *>(row) + k;
        if (n >= 8) {
            typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(1)));
            const words2 v = *reinterpret_cast<const words2 *>(p);
            w[0] = v.x;
            w[1] = v.y;
        } else {
            w[0] = w[1] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) w[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
        }
    }
    __device__ __forceinline__ void operands(long *b) const
    {
        const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), hi = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
        b[0] = (long)((uint64_t)lo | (uint64_t)hi << 32);
    }
};

// Four neighbouring results, `n` of which exist, to y[at] of one of the types.
__device__ __forceinline__ void store_four(void *y, int type, size_t at, f32x4 v, int n)
{
    if (type == XNOR_F32) {
        float *p = static_cast<float *>(y) + at;
        typedef float four __attribute__((ext_vector_type(4), aligned(4)));
        if (n >= 4) *reinterpret_cast<four *>(p) = v;
        else
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) p[i] = v[i];
        return;
    }
    typedef uint16_t halves __attribute__((ext_vector_type(4), aligned(2)));
    halves h;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = type == XNOR_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v[i]) : __builtin_bit_cast(uint16_t, (_Float16)v[i]);
    uint16_t *p = static_cast<uint16_t *>(y) + at;
    if (n >= 4) *reinterpret_cast<halves *>(p) = h;
    else
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) p[i] = h[i];
}

}  // namespace xnor
