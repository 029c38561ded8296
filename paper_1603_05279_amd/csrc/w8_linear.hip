// Products of 8-bit rows with 8-bit weights (contract: xnor_lowbit.h): few rows, and the choice of a kernel.
#include "xnor_internal.h"
#include "lowbit.h"
#include "w8_form.h"
#include "w8_choice.h"
#include "w8_linear.h"
#include <algorithm>
#include <cmath>

namespace xnor {

namespace {

// 16 * TILES rows x 16 outputs per workgroup, whose eight waves share the inputs in chunks of 128: a lane takes 32 neighbouring bytes of its row (lane & 15) and of its output,
// and the two instructions of 64 inputs their halves.
// What bounds it: the memory, and the launch: one row 9216 -> 4096 8.0 us, 38 MB, 4.7 TB/s; 16 rows 4096 -> 4096 6.5.
template <int TILES> __global__ __launch_bounds__(512) void w8_rows_kernel(W8Args a)
{
    constexpr int WAVES = 8, AT_ONCE = TILES == 1 ? 4 : TILES == 2 ? 3 : 2;
    __shared__ __attribute__((aligned(16))) int red[WAVES][TILES][64 * 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quarter = lane >> 4;
    const int row0 = blockIdx.y * 16 * TILES, out = blockIdx.x * 16 + col;
    const int8_t *x[TILES], *w = a.w + (size_t)min(out, a.out - 1) * a.in + 32 * quarter;
#pragma unroll
    for (int t = 0; t < TILES; ++t) x[t] = a.q + (size_t)min(row0 + 16 * t + col, a.rows - 1) * a.in + 32 * quarter;
    i32x4 acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = i32x4{0, 0, 0, 0};
    const int whole = a.in / 128;
    for (int c0 = wave; c0 < whole; c0 += WAVES * AT_ONCE) {
        i32x4 wv[AT_ONCE][2], xv[AT_ONCE][TILES][2];
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            const int c = c0 + n * WAVES;
            if (c >= whole) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                wv[n][i] = *reinterpret_cast<const i32x4_any *>(w + (size_t)c * 128 + 16 * i);
#pragma unroll
                for (int t = 0; t < TILES; ++t) xv[n][t][i] = *reinterpret_cast<const i32x4_any *>(x[t] + (size_t)c * 128 + 16 * i);
            }
        }
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            if (c0 + n * WAVES >= whole) break;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < TILES; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[n][i], xv[n][t][i], acc[t], 0, 0, 0);
        }
    }
    if (whole * 128 < a.in && whole % WAVES == wave) {
        const int k = whole * 128 + 32 * quarter;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const i32x4 wv = bytes16(w - 32 * quarter, k + 16 * i, a.in);
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, bytes16(x[t] - 32 * quarter, k + 16 * i, a.in), acc[t], 0, 0, 0);
        }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) *reinterpret_cast<i32x4 *>(&red[wave][t][4 * lane]) = acc[t];
    __syncthreads();
    if (wave >= TILES) return;
    i32x4 sum = *reinterpret_cast<const i32x4 *>(&red[0][wave][4 * lane]);
#pragma unroll
    for (int i = 1; i < WAVES; ++i) sum += *reinterpret_cast<const i32x4 *>(&red[i][wave][4 * lane]);
    const int o = blockIdx.x * 16 + 4 * quarter, row = row0 + 16 * wave + col;
    if (row >= a.rows || o >= a.out) return;
    const Split xs(a.x_scale[row]);
    f32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = min(o + i, a.out - 1);
        y[i] = scaled_sum(sum[i], xs, Split(a.w_scale[at])) + (a.bias ? a.bias[at] : 0.0f);
    }
    store_four(a.y, a.type, (size_t)row * a.out + o, y, a.out - o);
}

xnor_status launch_rows(W8Args a, int tiles, hipStream_t stream)
{
    const int rows = a.rows, most = 65535 * 16 * tiles;                 // (a launch's second dimension holds 65535 workgroups)
    for (int first = 0; first < rows; first += most) {
        a.rows = std::min(rows - first, most);
        const dim3 grid((unsigned)((a.out + 15) / 16), (unsigned)((a.rows + 16 * tiles - 1) / (16 * tiles)));
        if (tiles == 1) w8_rows_kernel<1><<<grid, dim3(512), 0, stream>>>(a);
        else if (tiles == 2) w8_rows_kernel<2><<<grid, dim3(512), 0, stream>>>(a);
        else w8_rows_kernel<4><<<grid, dim3(512), 0, stream>>>(a);
        if (xnor_status e = hip_status(hipGetLastError())) return e;
        a.q += (size_t)a.rows * a.in;
        a.x_scale += a.rows;
        a.y = static_cast<char *>(a.y) + (size_t)a.rows * a.out * type_bytes(a.type);
    }
    return XNOR_OK;
}

}  // namespace

bool w8_linear_needs(int rows, int in, int out) { return w8_choice(rows, in, out).shares > 1; }

size_t w8_linear_workspace_bytes(int rows, int in, int out) { return w8_share_bytes(rows, in, out); }

xnor_status launch_w8_linear(const int8_t *q, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, void *workspace, int rows,
                             int in, int out, int type, hipStream_t stream)
{
    const W8Args a{q, w, x_scale, w_scale, bias, y, workspace, rows, in, out, type};
    const W8Choice c = w8_choice(rows, in, out);
    return c.tiles ? launch_rows(a, c.tiles, stream) : launch_w8_tiles(a, c.side, c.shares, stream);
}

}  // namespace xnor
