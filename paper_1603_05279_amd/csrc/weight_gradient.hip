// Gradients of a product's weights and bias from the 8-bit rows that it read (contract: xnor_lowbit.h).
//
//     g_w[o][k] = sum_r g[r][o] x[r][k],    x = q * scale
// is a product of two matrices that both run along the rows, which neither stores next to each other.  Three launches:
//   range   the largest magnitude of every column of g (and its sum, the bias' gradient) and of the scales, in parts of the rows
//   stage   both matrices as float16 operands of the matrix instructions, transposed, each column multiplied by the power of two that brings its largest to 2^15 (float16
//           then holds 8- and 11-bit gradients exactly down to 2^-29 of the largest)
//   product the sums, and the powers of two taken out again
#include "xnor_internal.h"
#include "lowbit.h"
#include "w4_form.h"
#include <algorithm>

namespace xnor {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int STAGED_ROWS = 64, STAGED_COLS = 128;      // of a workgroup of the second launch

// Where the launches keep what they hand on:
//   x, g     [tile of 32 columns][step of 16 rows][part][lane][16 bytes]: lane holds column lane & 31, rows 8 (lane >> 5) .. + 7 of the step; rows behind the last are 0
//   top, sum [part of the rows][columns]: largest magnitudes of g and of the scales, sums of g
//   e        exponents of the columns of g and of the groups
struct Places {
    int steps, parts_x, parts_g, tiles_x, tiles_g, groups, parts, columns;
    size_t x_at, g_at, top_at, sum_at, e_at, total;
    __host__ __device__ Places(int rows, int in, int out, int group, int type, int w_type)
    {
        steps = (rows + STAGED_ROWS - 1) / STAGED_ROWS * (STAGED_ROWS / 16);
        parts_x = w_type == XNOR_BF16 ? 1 : 2;
        parts_g = w_type != XNOR_BF16 && type == XNOR_F32 ? 2 : 1;
        tiles_x = (in + 31) / 32;
        tiles_g = (out + 31) / 32;
        groups = group ? (in + group - 1) / group : 1;
        columns = (out + 3) / 4 * 4 + (groups + 3) / 4 * 4;     // (g's first, the groups from `groups_at` on)
        const int blocks = (out + 511) / 512 + (groups + 511) / 512, wanted = (512 + blocks - 1) / blocks, most = (rows + 31) / 32;
        parts = wanted < most ? wanted : most;
        x_at = 0;
        g_at = x_at + (size_t)tiles_x * steps * parts_x * 1024;
        top_at = g_at + (size_t)tiles_g * steps * parts_g * 1024;
        sum_at = top_at + (size_t)parts * columns * 4;
        e_at = sum_at + (size_t)parts * columns * 4;
        total = e_at + (size_t)columns * 4;
    }
    __host__ __device__ int groups_at(int out) const { return (out + 3) / 4 * 4; }
};

struct GradArgs {
    const int8_t *q;
    const float *scale;
    const void *g;
    void *g_w;
    float *g_bias;
    uint8_t *work;
    long long g_stride;
    int rows, in, out, group, type, w_type, accumulate;
};

// Largest finite magnitude and sum of 8 columns per lane; four waves take the rows of a part in turn.
template <int TYPE> __device__ __forceinline__ void range_of(const void *m, long long stride, int rows, int cols, int block, int part, int parts, uint32_t *top, float *sum)
{
    typedef real_t<TYPE> T;
    __shared__ uint32_t tops[4][512];
    __shared__ float sums[4][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = 512 * block + 8 * lane, n = cols - c;
    const int first = (int)((long long)rows * part / parts), last = (int)((long long)rows * (part + 1) / parts);
    uint32_t t[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int r = first + wave; r < last; r += 4) {
        Real8<TYPE> v;
        v.load(static_cast<const T *>(m) + (size_t)r * stride + c, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t bits = __float_as_uint(v[j]) & 0x7fffffffu;
            t[j] = max(t[j], bits < 0x7f800000u ? bits : 0u);
            s[j] += v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        tops[wave][8 * lane + j] = t[j];
        sums[wave][8 * lane + j] = s[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 512 && 512 * block + i < cols; i += 256) {
        top[512 * block + i] = max(max(tops[0][i], tops[1][i]), max(tops[2][i], tops[3][i]));
        if (sum) sum[512 * block + i] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    }
}

template <int TYPE> __global__ __launch_bounds__(256) void gradient_range_kernel(GradArgs a)
{
    const Places p(a.rows, a.in, a.out, a.group, a.type, a.w_type);
    const int blocks_g = (a.out + 511) / 512, part = blockIdx.y;
    uint32_t *top = reinterpret_cast<uint32_t *>(a.work + p.top_at) + (size_t)part * p.columns;
    float *sum = reinterpret_cast<float *>(a.work + p.sum_at) + (size_t)part * p.columns;
    if ((int)blockIdx.x < blocks_g) range_of<TYPE>(a.g, a.g_stride, a.rows, a.out, blockIdx.x, part, p.parts, top, sum);
    else range_of<XNOR_F32>(a.scale, p.groups, a.rows, p.groups, blockIdx.x - blocks_g, part, p.parts, top + p.groups_at(a.out), nullptr);
}

// 64 rows x 128 columns of one of the matrices, through LDS.
template <int TYPE> __global__ __launch_bounds__(256) void gradient_stage_kernel(GradArgs a)
{
    typedef real_t<TYPE> T;
    constexpr int PITCH = STAGED_COLS + 1;
    __shared__ float tile[STAGED_ROWS * PITCH];
    __shared__ int exponents[STAGED_COLS];
    const Places p(a.rows, a.in, a.out, a.group, a.type, a.w_type);
    const int blocks_g = (a.out + STAGED_COLS - 1) / STAGED_COLS, tid = threadIdx.x;
    const bool is_g = (int)blockIdx.x < blocks_g;
    const int c0 = STAGED_COLS * (is_g ? blockIdx.x : blockIdx.x - blocks_g), r0 = STAGED_ROWS * blockIdx.y, cols = is_g ? a.out : a.in;
    if (tid < STAGED_COLS && c0 + tid < cols) {
        const int at = is_g ? c0 + tid : p.groups_at(a.out) + (a.group ? (c0 + tid) / a.group : 0);
        const uint32_t *top = reinterpret_cast<const uint32_t *>(a.work + p.top_at) + at;
        uint32_t most = 0;
        for (int i = 0; i < p.parts; ++i) most = max(most, top[(size_t)i * p.columns]);
        const int e = __builtin_amdgcn_frexp_expf(__uint_as_float(most)) - (is_g ? 15 : 8);       // (an 8-bit number brings 2^7)
        exponents[tid] = e;
        if (r0 == 0) {
            reinterpret_cast<int *>(a.work + p.e_at)[at] = e;
            if (is_g && a.g_bias) {
                const float *sum = reinterpret_cast<const float *>(a.work + p.sum_at) + at;
                float s = 0.0f;
                for (int i = 0; i < p.parts; ++i) s += sum[(size_t)i * p.columns];
                a.g_bias[at] = a.accumulate ? a.g_bias[at] + s : s;
            }
        }
    }
    __syncthreads();
    const int c = 8 * (tid & 15);
#pragma unroll
    for (int i = 0; i < STAGED_ROWS / 16; ++i) {
        const int r = (tid >> 4) + 16 * i, n = r0 + r < a.rows ? cols - c0 - c : 0;
        float *to = tile + r * PITCH + c;
        if (is_g) {
            Real8<TYPE> v;
            v.load(static_cast<const T *>(a.g) + (size_t)(r0 + r) * a.g_stride + c0 + c, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) to[j] = j < n ? __builtin_amdgcn_ldexpf(v[j], -exponents[c + j]) : 0.0f;
        } else {
            Eight<ROWS_I8> v;
            v.load(a.q + (size_t)(r0 + r) * a.in + c0, c, n);
            const float s = n > 0 ? a.scale[(size_t)(r0 + r) * p.groups + (a.group ? (c0 + c) / a.group : 0)] : 0.0f;
            const float scaled = n > 0 ? __builtin_amdgcn_ldexpf(s, -exponents[c]) : 0.0f;       // (eight columns are of one group)
#pragma unroll
            for (int j = 0; j < 8; ++j) to[j] = j < n ? (float)(int8_t)(v.w[j / 4] >> (8 * (j & 3))) * scaled : 0.0f;
        }
    }
    __syncthreads();
    const int parts = is_g ? p.parts_g : p.parts_x, tiles = is_g ? p.tiles_g : p.tiles_x;
    u32x4 *to = reinterpret_cast<u32x4 *>(a.work + (is_g ? p.g_at : p.x_at));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int unit = tid + 256 * i, lane = unit & 63, step = unit >> 6 & 3, t = unit >> 8;       // (tile of the four, step of the four)
        if (c0 / 32 + t >= tiles) break;
        const float *from = tile + (16 * step + 8 * (lane >> 5)) * PITCH + 32 * t + (lane & 31);
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = from[j * PITCH];
            hi[j] = (_Float16)v;
            const float rest = v - (float)hi[j];
            lo[j] = (_Float16)(__builtin_fabsf(v) < __builtin_inff() ? rest : 0.0f);
        }
        u32x4 *at = to + (((size_t)(c0 / 32 + t) * p.steps + r0 / 16 + step) * parts) * 64 + lane;
        at[0] = __builtin_bit_cast(u32x4, hi);
        if (parts == 2) at[64] = __builtin_bit_cast(u32x4, lo);
    }
}

// A wave makes 64 columns of x by 64 of g, a workgroup 128 x 128, operands straight from what was staged.
template <int PX, int PG> __global__ __launch_bounds__(256) void gradient_product_kernel(GradArgs a)
{
    const Places p(a.rows, a.in, a.out, a.group, a.type, a.w_type);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tx = blockIdx.x * 4 + (wave & 1) * 2, tg = blockIdx.y * 4 + (wave >> 1) * 2;
    const f16x8 *x[2], *g[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i] = reinterpret_cast<const f16x8 *>(a.work + p.x_at) + (size_t)min(tx + i, p.tiles_x - 1) * p.steps * PX * 64 + lane;
        g[i] = reinterpret_cast<const f16x8 *>(a.work + p.g_at) + (size_t)min(tg + i, p.tiles_g - 1) * p.steps * PG * 64 + lane;
    }
    f32x16 acc[2][2] = {};
    for (int s = 0; s < p.steps; ++s) {
        f16x8 av[2][PX], bv[2][PG];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 0; k < PX; ++k) av[i][k] = x[i][((size_t)s * PX + k) * 64];
#pragma unroll
            for (int k = 0; k < PG; ++k) bv[i][k] = g[i][((size_t)s * PG + k) * 64];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av[i][0], bv[j][0], acc[i][j], 0, 0, 0);
                if (PX == 2) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av[i][PX - 1], bv[j][0], acc[i][j], 0, 0, 0);
                if (PG == 2) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av[i][0], bv[j][PG - 1], acc[i][j], 0, 0, 0);
            }
    }
    const int *e = reinterpret_cast<const int *>(a.work + p.e_at);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int o = 32 * (tg + j) + (lane & 31);
        if (o >= a.out) continue;
        const int eg = e[o];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int k = 32 * (tx + i) + 8 * b + 4 * (lane >> 5), n = a.in - k;
                if (n <= 0) continue;
                const int ex = e[p.groups_at(a.out) + (a.group ? k / a.group : 0)] + eg;
                const size_t at = (size_t)o * a.in + k;
                f32x4 v;
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    v[m] = __builtin_amdgcn_ldexpf(acc[i][j][4 * b + m], ex);
                    if (a.accumulate && m < n)
                        v[m] += a.w_type == XNOR_F32    ? static_cast<const float *>(a.g_w)[at + m]
                                : a.w_type == XNOR_BF16 ? (float)static_cast<const __bf16 *>(a.g_w)[at + m]
                                                        : (float)static_cast<const _Float16 *>(a.g_w)[at + m];
                }
                store_four(a.g_w, a.w_type, at, v, n);
            }
    }
}

__global__ __launch_bounds__(256) void gradient_zero_kernel(void *g_w, float *g_bias, size_t words, bool odd, int out)
{
    const size_t step = (size_t)gridDim.x * 256, first = (size_t)blockIdx.x * 256 + threadIdx.x;
    for (size_t i = first; i < words; i += step) static_cast<uint32_t *>(g_w)[i] = 0;
    if (odd && first == 0) static_cast<uint16_t *>(g_w)[2 * words] = 0;
    if (g_bias)
        for (size_t i = first; i < (size_t)out; i += step) g_bias[i] = 0.0f;
}

}  // namespace

size_t weight_gradient_workspace_bytes(int rows, int in, int out, int group, int type, int w_type) { return Places(rows, in, out, group, type, w_type).total; }

xnor_status launch_weight_gradient(const int8_t *q, const float *scale, const void *g_y, long long g_stride, void *g_w, float *g_bias, int accumulate,
                                   void *workspace, int rows, int in, int out, int group, int type, int w_type, hipStream_t stream)
{
    if (rows == 0) {
        const size_t bytes = (size_t)in * out * type_bytes(w_type);
        gradient_zero_kernel<<<dim3(2048), dim3(256), 0, stream>>>(g_w, g_bias, bytes / 4, bytes % 4 != 0, out);
        return hip_status(hipGetLastError());
    }
    const GradArgs a{q, scale, g_y, g_w, g_bias, static_cast<uint8_t *>(workspace), g_stride, rows, in, out, group, type, w_type, accumulate};
    const Places p(rows, in, out, group, type, w_type);
    if ((rows + STAGED_ROWS - 1) / STAGED_ROWS > 65535 || (p.tiles_g + 3) / 4 > 65535) return XNOR_ERR_SHAPE;
    const dim3 range((unsigned)((out + 511) / 512 + (p.groups + 511) / 512), (unsigned)p.parts);
    const dim3 stage((unsigned)((out + STAGED_COLS - 1) / STAGED_COLS + (in + STAGED_COLS - 1) / STAGED_COLS), (unsigned)(p.steps / 4));
    const dim3 product((unsigned)((p.tiles_x + 3) / 4), (unsigned)((p.tiles_g + 3) / 4));
    xnor_status status = XNOR_OK;
    by_type(type, [&](auto t) {
        gradient_range_kernel<t()><<<range, dim3(256), 0, stream>>>(a);
        status = hip_status(hipGetLastError());
        if (status) return;
        gradient_stage_kernel<t()><<<stage, dim3(256), 0, stream>>>(a);
        status = hip_status(hipGetLastError());
    });
    if (status) return status;
    if (p.parts_x == 1) gradient_product_kernel<1, 1><<<product, dim3(256), 0, stream>>>(a);
    else if (p.parts_g == 1) gradient_product_kernel<2, 1><<<product, dim3(256), 0, stream>>>(a);
    else gradient_product_kernel<2, 2><<<product, dim3(256), 0, stream>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace xnor
