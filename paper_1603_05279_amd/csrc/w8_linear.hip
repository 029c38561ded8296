// Products of 8-bit rows with 8-bit weights (contract: xnor_lowbit.h).
#include "xnor_internal.h"
#include "lowbit.h"
#include "w4_form.h"
#include "w8_form.h"
#include <algorithm>

namespace xnor {

namespace {

struct W8Args {
    const int8_t *q, *w;
    const float *x_scale, *w_scale, *bias;
    void *y;
    int rows, in, out, type;
};

// 16 rows x 16 outputs per workgroup, whose eight waves share the inputs in chunks of 128: a lane takes 32 neighbouring bytes of its row (lane & 15) and of its output, and
// the two instructions of 64 inputs their halves.
__global__ __launch_bounds__(512) void w8_rows_kernel(W8Args a)
{
    constexpr int WAVES = 8;
    __shared__ __attribute__((aligned(16))) int red[WAVES][64 * 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const int row = blockIdx.y * 16 + col, out = blockIdx.x * 16 + col;
    const int8_t *x = a.q + (size_t)min(row, a.rows - 1) * a.in, *w = a.w + (size_t)min(out, a.out - 1) * a.in;
    i32x4 acc{0, 0, 0, 0};
    for (int k = 128 * wave + 32 * quarter; k - 32 * quarter < a.in; k += 128 * WAVES) {
        i32x4 av[2], bv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            av[i] = bytes16(w, k + 16 * i, a.in);
            bv[i] = bytes16(x, k + 16 * i, a.in);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[i], bv[i], acc, 0, 0, 0);
    }
    *reinterpret_cast<i32x4 *>(&red[wave][4 * lane]) = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) acc += *reinterpret_cast<const i32x4 *>(&red[i][4 * lane]);
    const int o = blockIdx.x * 16 + 4 * quarter;
    if (row >= a.rows || o >= a.out) return;
    const Split xs(a.x_scale[row]);
    f32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = min(o + i, a.out - 1);
        y[i] = scaled_sum(acc[i], xs, Split(a.w_scale[at])) + (a.bias ? a.bias[at] : 0.0f);
    }
    store_four(a.y, a.type, (size_t)row * a.out + o, y, a.out - o);
}

}  // namespace

size_t w8_linear_workspace_bytes(int, int, int) { return 0; }
bool w8_linear_needs(int, int, int) { return false; }

xnor_status launch_w8_linear(const int8_t *q, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, void *, int rows, int in,
                             int out, int type, hipStream_t stream)
{
    const W8Args a{q, w, x_scale, w_scale, bias, y, rows, in, out, type};
    // (a launch's second dimension holds 65535 workgroups)
    for (int first = 0; first < rows; first += 65535 * 16) {
        W8Args part = a;
        part.q += (size_t)first * in;
        part.x_scale += first;
        part.y = static_cast<char *>(y) + (size_t)first * out * type_bytes(type);
        part.rows = std::min(rows - first, 65535 * 16);
        w8_rows_kernel<<<dim3((unsigned)((out + 15) / 16), (unsigned)((part.rows + 15) / 16)), dim3(512), 0, stream>>>(part);
        if (xnor_status e = hip_status(hipGetLastError())) return e;
    }
    return XNOR_OK;
}

}  // namespace xnor
