// The image of 4-bit weights that the products read: codes in the order of the matrix instructions' operands, then the groups' scales and
// zero points in the order of their results.
//   codes  [tile of 16 outputs][chunk of 128 inputs][lane 0..63][word 0..3]: word j of a lane holds output lane & 15, inputs
//          32 j + 8 (lane >> 4) .. + 7 of the chunk, an even one e at bit 2 e, an odd one at bit 16 + 2 (e - 1), so that a mask takes a pair
//          (0, 1), (2, 3) .. out of the two halves of a word; a wave reads 1 KB in one piece
//   scale  [tile][group][output 0..15] float32, 0 past the last output
//   zero   [tile][group][output 0..15] bytes
#pragma once
#include <stddef.h>
#include <hip/hip_runtime.h>

namespace xnor {

struct W4Layout {
    int tiles, chunks, groups;
    __host__ __device__ W4Layout(int out, int in, int group) : tiles((out + 15) / 16), chunks((in + 127) / 128), groups((in + group - 1) / group) {}
    __host__ __device__ size_t scale_at() const { return (size_t)tiles * chunks * 1024; }
    __host__ __device__ size_t zero_at() const { return scale_at() + (size_t)tiles * groups * 64; }
    __host__ __device__ size_t bytes() const { return zero_at() + (size_t)tiles * groups * 16; }
};

}  // namespace xnor
