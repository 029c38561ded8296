// Bytes as operands of the 8-bit matrix instructions, and their sums under two scales.
#pragma once
#include "w4_form.h"

namespace xnor {

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef i32x4 i32x4_any __attribute__((aligned(1)));

// Bytes k .. k + 15 of a row of `in`, 0 behind its end; the row starts at any address (the memory takes such accesses whole).  Past the end: the row's last 16, moved down.
__device__ __forceinline__ i32x4 bytes16(const int8_t *row, int k, int in)
{
    const int past = k + 16 - in;
    if (past <= 0) return *reinterpret_cast<const i32x4_any *>(row + k);
    i32x4 v{0, 0, 0, 0};
    if (past >= 16) return v;
    if (in < 16) {
        for (int i = 0; i < 16 - past; ++i) {
            const uint32_t b = (uint32_t)(uint8_t)row[k + i] << (8 * (i & 3));
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] |= i / 4 == w ? (int)b : 0;
        }
        return v;
    }
    const i32x4 last = *reinterpret_cast<const i32x4_any *>(row + in - 16);
    const int words = past >> 2;
    uint32_t w[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        w[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i] = j == i + words ? (uint32_t)last[j] : w[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (int)__builtin_amdgcn_alignbyte(w[i + 1], w[i], past & 3);
    return v;
}

// A scale as mantissa and exponent, so that the product of two neither overflows nor vanishes before it meets the sum.
struct Split {
    float mantissa;
    int exponent;
    __device__ __forceinline__ explicit Split(float s) : mantissa(__builtin_amdgcn_frexp_mantf(s)), exponent(__builtin_amdgcn_frexp_expf(s)) {}
};
__device__ __forceinline__ float scaled_sum(int sum, const Split &x, float w_mantissa, int w_exponent)
{
    return __builtin_amdgcn_ldexpf((float)sum * (x.mantissa * w_mantissa), x.exponent + w_exponent);
}
__device__ __forceinline__ float scaled_sum(int sum, const Split &x, const Split &w) { return scaled_sum(sum, x, w.mantissa, w.exponent); }

}  // namespace xnor
