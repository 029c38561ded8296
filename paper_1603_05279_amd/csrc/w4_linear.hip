// Products of rows with 4-bit weights under group scales (contracts: xnor_lowbit.h).
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"
#include "w4_form.h"
#include "w4_image.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr float TINY = 0x1p-100f;

// ---- weights: real numbers to codes, codes to the image ---------------------------------------------------------------

// A thread rounds eight neighbouring weights of a row; the 4, 8 or 16 lanes of a group exchange its extremes.  One row per workgroup.
template <int TYPE>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const void *w, long long stride, uint32_t *codes, float *scale, uint8_t *zero, int in,
                                                          int group)
{
    typedef real_t<TYPE> T;
    const size_t row = blockIdx.x;
    const int eights = (in + 31) / 32 * 4, groups = (in + group - 1) / group, lanes = group / 8;
    for (int e0 = 0; e0 < eights; e0 += blockDim.x) {           // (whole waves: lanes past the row hold zeros)
        const int e = e0 + threadIdx.x, c = 8 * e;
        Real8<TYPE> v;
        v.load(static_cast<const T *>(w) + row * (size_t)stride + c, in - c);
        float lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo = fminf(lo, v[j]);
            hi = fmaxf(hi, v[j]);
        }
        for (int s = lanes / 2; s > 0; s >>= 1) {
            lo = fminf(lo, __shfl_xor(lo, s, 64));
            hi = fmaxf(hi, __shfl_xor(hi, s, 64));
        }
        const float span = zero ? hi - lo : fmaxf(hi, -lo), levels = zero ? 15.0f : 7.0f;
        const bool some = span >= TINY;
        const float inverse = some ? levels / span : 0.0f;
        const float z = zero ? __builtin_rintf(-lo * inverse) : 8.0f;
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float u = fminf(fmaxf(__builtin_rintf(v[j] * inverse) + z, 0.0f), 15.0f);
            word |= (uint32_t)u << (4 * j);
        }
        if (e < eights) codes[row * eights + e] = word;
        if (c < in && e % lanes == 0) {
            scale[row * groups + c / group] = some ? span / levels : 0.0f;
            if (zero) zero[row * groups + c / group] = (uint8_t)z;
        }
    }
}

// One thread per 32-bit word of the image, then per scale and zero point.
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint32_t *codes, const float *scale, const uint8_t *zero, uint8_t *image, int out, int in,
                                                      int group)
{
    const W4Layout l(out, in, group);
    const size_t words = l.scale_at() / 4, factors = (size_t)l.tiles * l.groups * 16;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < words) {
        const int j = (int)(i & 3), lane = (int)(i >> 2 & 63);
        const size_t block = i >> 8;
        const int chunk = (int)(block % l.chunks), o = (int)(block / l.chunks) * 16 + (lane & 15), k = 128 * chunk + 32 * j + 8 * (lane >> 4);
        const int eights = (in + 31) / 32 * 4;
        uint32_t word = 0;
        if (o < out && k < 8 * eights) {
            const uint32_t c = codes[(size_t)o * eights + k / 8];
#pragma unroll
            for (int e = 0; e < 8; ++e) word |= (c >> (4 * e) & 15u) << (4 * (e / 2 + 4 * (e & 1)));
        }
        reinterpret_cast<uint32_t *>(image)[i] = word;
    } else if (i < words + factors) {
        const size_t f = i - words;
        const int o = (int)(f / ((size_t)l.groups * 16)) * 16 + (int)(f & 15), g = (int)(f / 16 % l.groups);
        reinterpret_cast<float *>(image + l.scale_at())[f] = o < out ? scale[(size_t)o * l.groups + g] : 0.0f;
        image[l.zero_at() + f] = o < out && zero ? zero[(size_t)o * l.groups + g] : 8;
    }
}

// ---- products -----------------------------------------------------------------------------------------------------------

struct W4Args {
    const void *x;
    const float *x_scale;
    const uint8_t *image;
    void *y;
    long long x_stride;             // in elements
    int rows, in, out, group, x_group, x_groups;
};

// A workgroup makes 16 outputs of 16 * BLOCKS rows; its waves take every WAVES-th chunk of 128 inputs and add their sums in LDS.  Nothing is
// staged: a code is read once, straight from the image into the lane that multiplies it.
template <int X, int YTYPE, int BLOCKS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void w4_rows_kernel(W4Args a)
{
    typedef Form<X> F;
    typedef real_t<YTYPE> Y;
    __shared__ __attribute__((aligned(16))) float red[WAVES][16 * BLOCKS][20];
    const W4Layout l(a.out, a.in, a.group);
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = blockIdx.x, row0 = blockIdx.y * 16 * BLOCKS;
    const u32x4 *codes = reinterpret_cast<const u32x4 *>(a.image) + (size_t)tile * l.chunks * 64 + lane;
    const float *scales = reinterpret_cast<const float *>(a.image + l.scale_at()) + (size_t)tile * l.groups * 16 + 4 * quarter;
    const uint8_t *zeros = a.image + l.zero_at() + (size_t)tile * l.groups * 16 + (X == ROWS_I8 ? col : 4 * quarter);
    const char *xrow[BLOCKS];
    bool real[BLOCKS];
    constexpr int XBYTES = X == ROWS_F32 ? 4 : X == ROWS_I8 ? 1 : 2;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        const int row = row0 + 16 * b + col;
        real[b] = row < a.rows;
        xrow[b] = static_cast<const char *>(a.x) + (size_t)(real[b] ? row : 0) * a.x_stride * XBYTES;
    }
    f32x4 total[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) total[b] = f32x4{0, 0, 0, 0};
    const int steps_per_group = a.group / 32;
    for (int chunk = wave; chunk < l.chunks; chunk += WAVES) {
        const u32x4 w = codes[(size_t)chunk * 64];
        Eight<X> x[4][BLOCKS];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const int k = 128 * chunk + 32 * j + 8 * quarter;
                x[j][b].load(xrow[b], k, real[b] ? a.in - k : 0);
            }
        typename F::acc_t acc[BLOCKS], sum[BLOCKS];
        uint32_t zero = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k0 = 128 * chunk + 32 * j, g = min(k0 / a.group, l.groups - 1);
            if (j % steps_per_group == 0) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) acc[b] = sum[b] = typename F::acc_t{0, 0, 0, 0};
                if (X == ROWS_I8) zero = zeros[(size_t)g * 16] * 0x01010101u;
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                typename F::operand_t xo[F::PARTS];
                x[j][b].operands(xo);
                if constexpr (X == ROWS_I8) {
                    acc[b] = F::mfma(F::widen(w[j], zero), xo[0], acc[b]);
                } else {
#pragma unroll
                    for (int p = 0; p < F::PARTS; ++p) {
                        acc[b] = F::mfma(F::widen(w[j]), xo[p], acc[b]);
                        sum[b] = F::mfma(F::ones(), xo[p], sum[b]);
                    }
                }
            }
            if ((j + 1) % steps_per_group == 0) {           // (a group past the last input has sums of zero)
                const f32x4 s = *reinterpret_cast<const f32x4 *>(scales + (size_t)g * 16);
                uint32_t z = 0;
                if constexpr (X != ROWS_I8) z = *reinterpret_cast<const uint32_t *>(zeros + (size_t)g * 16);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    float xs = 1.0f;
                    if (X == ROWS_I8 && a.x_group)
                        xs = a.x_scale[(size_t)min(row0 + 16 * b + col, a.rows - 1) * a.x_groups + min(k0 / a.x_group, a.x_groups - 1)];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float part;
                        if constexpr (X == ROWS_I8) part = (float)acc[b][v] * xs;
                        else part = __builtin_fmaf(-(F::OFFSET + (float)(z >> (8 * v) & 255u)), sum[b][v], acc[b][v]);
                        total[b][v] = __builtin_fmaf(s[v], part, total[b][v]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) *reinterpret_cast<f32x4 *>(&red[wave][16 * b + col][4 * quarter]) = total[b];
    __syncthreads();
    for (int i = tid; i < 64 * BLOCKS; i += 64 * WAVES) {
        const int r = i >> 2, q = i & 3, row = row0 + r, o = 16 * tile + 4 * q;
        f32x4 s = *reinterpret_cast<const f32x4 *>(&red[0][r][4 * q]);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += *reinterpret_cast<const f32x4 *>(&red[w][r][4 * q]);
        if (row >= a.rows) continue;
        if (X == ROWS_I8 && !a.x_group) s *= a.x_scale[row];
        Y *y = static_cast<Y *>(a.y) + (size_t)row * a.out + o;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (o + v < a.out) y[v] = (Y)s[v];
    }
}

template <int X, int YTYPE> void launch_rows(const W4Args &a, hipStream_t stream)
{
    const unsigned tiles = (unsigned)((a.out + 15) / 16);
    if (a.rows <= 16) w4_rows_kernel<X, YTYPE, 1, 8><<<dim3(tiles, 1), dim3(512), 0, stream>>>(a);
    else if (a.rows <= 32) w4_rows_kernel<X, YTYPE, 2, 8><<<dim3(tiles, 1), dim3(512), 0, stream>>>(a);
    else w4_rows_kernel<X, YTYPE, 4, 8><<<dim3(tiles, (unsigned)((a.rows + 63) / 64)), dim3(512), 0, stream>>>(a);
}

}  // namespace

size_t w4_wimg_bytes(int out, int in, int group) { return W4Layout(out, in, group).bytes(); }

xnor_status launch_w4_quantize(const void *w, long long stride, uint8_t *codes, float *scale, uint8_t *zero, int out, int in, int group, int type,
                               hipStream_t stream)
{
    const int eights = (in + 31) / 32 * 4, threads = std::min(256, (eights + 63) / 64 * 64);
    by_type(type, [&](auto t) {
        w4_quantize_kernel<t()><<<dim3((unsigned)out), dim3((unsigned)threads), 0, stream>>>(w, stride, reinterpret_cast<uint32_t *>(codes), scale, zero,
                                                                                             in, group);
    });
    return hip_status(hipGetLastError());
}

xnor_status launch_w4_pack(const uint8_t *codes, const float *scale, const uint8_t *zero, void *wimg, int out, int in, int group, hipStream_t stream)
{
    const W4Layout l(out, in, group);
    const size_t items = l.scale_at() / 4 + (size_t)l.tiles * l.groups * 16;
    w4_pack_kernel<<<dim3((unsigned)((items + 255) / 256)), dim3(256), 0, stream>>>(reinterpret_cast<const uint32_t *>(codes), scale, zero,
                                                                                    static_cast<uint8_t *>(wimg), out, in, group);
    return hip_status(hipGetLastError());
}

size_t w4_linear_workspace_bytes(int rows, int in, int out, int group)
{
    return w4_tiles_applies(rows) ? w4_tiles_workspace_bytes(rows, in, out, group) : 0;
}

xnor_status launch_w4_linear(const void *x, long long x_stride, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group, int type,
                             hipStream_t stream)
{
    if (w4_tiles_applies(rows)) return launch_w4_tiles(x, x_stride, nullptr, wimg, y, workspace, rows, in, out, group, 0, type, type, stream);
    const W4Args a{x, nullptr, static_cast<const uint8_t *>(wimg), y, x_stride, rows, in, out, group, 0, 1};
    by_type(type, [&](auto t) { launch_rows<t(), t()>(a, stream); });
    return hip_status(hipGetLastError());
}

xnor_status launch_w4_linear_q8(const int8_t *q, const float *x_scale, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group,
                                int x_group, int type, hipStream_t stream)
{
    if (w4_tiles_applies(rows)) return launch_w4_tiles(q, in, x_scale, wimg, y, workspace, rows, in, out, group, x_group, ROWS_I8, type, stream);
    const W4Args a{q, x_scale, static_cast<const uint8_t *>(wimg), y, in, rows, in, out, group, x_group, x_group ? (in + x_group - 1) / x_group : 1};
    by_type(type, [&](auto t) { launch_rows<ROWS_I8, t()>(a, stream); });
    return hip_status(hipGetLastError());
}

}  // namespace xnor
