// Bytes as operands of the 8-bit matrix instructions, and their sums under two scales.
#pragma once
#include "w4_form.h"

namespace xnor {

typedef i32x4 i32x4_any __attribute__((aligned(1)));

// Bytes k .. k + 15 of a row of `in`, 0 behind its end; the row starts at any address (the memory takes such accesses whole).
__device__ __forceinline__ i32x4 bytes16(const int8_t *row, int k, int in)
{
    if (k + 16 <= in) return *reinterpret_cast<const i32x4_any *>(row + k);
    i32x4 v{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k + i < in) v[i / 4] |= (int)((uint32_t)(uint8_t)row[k + i] << (8 * (i & 3)));
    return v;
}

// A scale as mantissa and exponent, so that the product of two neither overflows nor vanishes before it meets the sum.
struct Split {
    float mantissa;
    int exponent;
    __device__ __forceinline__ explicit Split(float s) : mantissa(__builtin_amdgcn_frexp_mantf(s)), exponent(__builtin_amdgcn_frexp_expf(s)) {}
};
__device__ __forceinline__ float scaled_sum(int sum, const Split &x, const Split &w)
{
    return __builtin_amdgcn_ldexpf((float)sum * (x.mantissa * w.mantissa), x.exponent + w.exponent);
}

}  // namespace xnor
