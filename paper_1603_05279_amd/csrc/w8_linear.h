// The product of 8-bit rows with 8-bit weights, as its kernels get it.
#pragma once
#include <hip/hip_runtime.h>
#include "xnor_lowbit.h"

namespace xnor {

struct W8Args {
    const int8_t *q, *w;
    const float *x_scale, *w_scale, *bias;
    void *y, *work;
    int rows, in, out, type;
};

// side: W8_LARGE or W8_SMALL; shares (of the inputs, W8_SMALL only): that many times rows x out sums of 32 bits, in whole tiles, in a.work
xnor_status launch_w8_tiles(const W8Args &a, int side, int shares, hipStream_t stream);

}  // namespace xnor
