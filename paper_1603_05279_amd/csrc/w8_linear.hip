// Products of 8-bit rows with 8-bit weights (contract: xnor_lowbit.h): few rows, and the choice of a kernel.
#include "xnor_internal.h"
#include "lowbit.h"
#include "w8_form.h"
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

// Which kernel takes a product: the shortest of their times in us, fitted to 150 products (inputs 256 to 9216, outputs 256 to 8192, 1 to 2048 rows, half of them no multiple of
// anything).
struct Choice {
    int tiles, side, shares;        // w8_rows_kernel's row tiles, or the side of w8_tiles.hip's tiles and the shares of the inputs
    double time;
};

double blocks(int n, int side) { return std::ceil((double)n / side); }

// w8_rows_kernel reads every weight once per 16, 32 or 64 rows and splits the inputs over its waves.  One, two and four tiles: 16 rows 9216 -> 4096 10.6, 11.5, 13.6; 32 rows
// 4096 -> 4096 10.0, 8.1, 9.2; 64 rows 17, 13.5, 11.7 (128 x 128 in four shares 15).  Rows that start between words of 32 bits: 15 rows 6086 -> 7076 31 (in shares 24).
Choice by_rows(int rows, int in, int out)
{
    const double turns = std::ceil(std::ceil(in / 128.0) / 8);
    Choice best{0, 0, 1, 0.0};
    for (int tiles : {1, 2, 4}) {
        const double n = blocks(out, 16) * blocks(rows, 16 * tiles) / 256;
        const double time = 4.3 + (tiles == 1 ? 0.85 : tiles == 2 ? 1.2 : 2.05) * (in % 4 ? 2.4 : 1.0) * turns * std::max(n, 0.7);
        if (best.tiles == 0 || time < best.time) best = {tiles, 0, 1, time};
    }
    return best;
}
// Tiles of 128 x 128: what a CU gets out of L2 bounds a chunk, 0.65 us for 256 workgroups (12 TB/s), and its way there and back where there are fewer.  In shares of the inputs
// where that fills the chip, which costs another launch and the sums' way through memory.  256 rows 9216 -> 4096 in 1, 2, 3, 4 and 6 shares 39, 26, 24, 26, 28; 512 rows
// 4096 -> 4096 in 1 and 2 21, 25.
Choice by_small_tiles(int row_blocks, int in, int out)
{
    const double chunks = std::ceil(in / 128.0), tiles = (double)row_blocks * blocks(out, W8_SMALL);
    Choice best{0, W8_SMALL, 0, 0.0};
    for (int shares : {1, 2, 3, 4, 6, 8}) {
        const double n = tiles * shares / 256;
        if (shares > 1 && (n > 2 || chunks < 2 * shares)) break;
        const double chunk = in % 16 == 0 ? std::max(0.48, 0.65 * n) : in % 4 == 0 ? std::max(0.85, 0.85 * n) : std::max(1.25, 0.95 * n);
        const double time = 4.0 + chunk * std::ceil(chunks / shares) + (shares > 1 ? 2.5 + 0.026 * tiles * shares : 0.0) + 0.002 * tiles;
        if (best.shares == 0 || time < best.time) best = {0, W8_SMALL, shares, time};
    }
    return best;
}
// Tiles of 256 x 256 take half as much out of L2 per result, one workgroup to a CU.  2048 rows 4096 -> 8192 83 us, in tiles of 128 x 128 91; 4096 rows 158, 175; 1024 rows 70, 45.
Choice by_large_tiles(int rows, int in, int out)
{
    const double tiles = blocks(rows, W8_LARGE) * blocks(out, W8_LARGE), rounds = std::ceil(tiles / 256);
    return {0, W8_LARGE, 1, 12 + (tiles <= 128 ? 0.85 : 1.06) * std::ceil(in / 64.0) * rounds * (in % 4 ? 1.5 : in % 16 ? 1.3 : 1.0) + 0.012 * tiles};
}
Choice choose(int rows, int in, int out)
{
    Choice best = by_rows(rows, in, out);
    for (const Choice &c : {by_small_tiles((int)blocks(rows, W8_SMALL), in, out), by_large_tiles(rows, in, out)})
        if (c.time < best.time) best = c;
    return best;
}
size_t share_bytes(int row_blocks, int in, int out)
{
    const int shares = by_small_tiles(row_blocks, in, out).shares;
    return shares > 1 ? (size_t)shares * row_blocks * (size_t)blocks(out, W8_SMALL) * W8_SMALL * W8_SMALL * 4 : 0;
}

}  // namespace

bool w8_linear_needs(int rows, int in, int out) { return choose(rows, in, out).shares > 1; }

// (the most of any number of rows up to this one: more than 512 tiles are not shared)
size_t w8_linear_workspace_bytes(int rows, int in, int out)
{
    size_t most = 0;
    for (int b = 1; b <= (int)blocks(rows, W8_SMALL) && b * blocks(out, W8_SMALL) <= 512; ++b) most = std::max(most, share_bytes(b, in, out));
    return most;
}

xnor_status launch_w8_linear(const int8_t *q, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, void *workspace, int rows,
                             int in, int out, int type, hipStream_t stream)
{
    const W8Args a{q, w, x_scale, w_scale, bias, y, workspace, rows, in, out, type};
    const Choice c = choose(rows, in, out);
    return c.tiles ? launch_rows(a, c.tiles, stream) : launch_w8_tiles(a, c.side, c.shares, stream);
}

}  // namespace xnor
