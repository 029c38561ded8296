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
constexpr unsigned MOST_GROUPS = 1u << 20;      // workgroups of a launch over weights, which may be more than 2^32 threads' worth

// ---- weights: real numbers to codes, codes to the image ---------------------------------------------------------------

// A thread rounds eight neighbouring weights of a row; the 4, 8 or 16 lanes of a group exchange its extremes.  One row per workgroup and turn.
// What bounds it: the memory (32000 x 4096 bfloat16 85 us, 3.9 TB/s).
template <int TYPE>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const void *w, long long stride, uint32_t *codes, float *scale, uint8_t *zero, int out,
                                                          int in, int group)
{
    typedef real_t<TYPE> T;
    const int eights = (in + 31) / 32 * 4, groups = (in + group - 1) / group, lanes = group / 8;
    for (size_t row = blockIdx.x; row < (size_t)out; row += gridDim.x)
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
            // (halves of both: the span of float32's largest of either sign is not a float32 number)
            const float span = zero ? 0.5f * hi - 0.5f * lo : 0.5f * fmaxf(hi, -lo), levels = zero ? 7.5f : 3.5f;
            const bool some = span >= 0.5f * TINY;
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

// Every other of eight codes, the lowest first, side by side in 16 bits.
__device__ __forceinline__ uint32_t every_other(uint32_t c)
{
    c &= 0x0f0f0f0fu;
    c = (c | c >> 4) & 0x00ff00ffu;
    return (c | c >> 8) & 0x0000ffffu;
}

// A lane's 16 bytes of the image per thread and turn, then a scale and zero point; once per layer.  What bounds it: the memory, read in pieces of 4 bytes
// (32000 x 4096 38 us, 3.7 TB/s; a word per thread 45).
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint32_t *codes, const float *scale, const uint8_t *zero, uint8_t *image, int out, int in,
                                                      int group)
{
    const W4Layout l(out, in, group);
    const size_t lanes = l.scale_at() / 16, factors = (size_t)l.tiles * l.groups * 16;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < lanes + factors; i += (size_t)gridDim.x * 256) {
        if (i < lanes) {
            const int lane = (int)(i & 63);
            const size_t block = i >> 6;
            const int chunk = (int)(block % l.chunks), o = (int)(block / l.chunks) * 16 + (lane & 15), eights = (in + 31) / 32 * 4;
            u32x4 words{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int eight = 16 * chunk + 4 * j + (lane >> 4);
                if (o < out && eight < eights) words[j] = codes[(size_t)o * eights + eight];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) words[j] = every_other(words[j]) | every_other(words[j] >> 4) << 16;
            reinterpret_cast<u32x4 *>(image)[i] = words;
        } else {
            const size_t f = i - lanes;
            const int o = (int)(f / ((size_t)l.groups * 16)) * 16 + (int)(f & 15), g = (int)(f / 16 % l.groups);
            reinterpret_cast<float *>(image + l.scale_at())[f] = o < out ? scale[(size_t)o * l.groups + g] : 0.0f;
            image[l.zero_at() + f] = o < out && zero ? zero[(size_t)o * l.groups + g] : 8;
        }
    }
}

// ---- products -----------------------------------------------------------------------------------------------------------

struct W4Args {
    const void *x;
    const float *x_scale;
    const uint8_t *image;
    void *y;
    long long x_stride;             // in elements
    int rows, in, out, x_groups, x_shift, type;     // a group's scale of x: group >> x_shift
};

// What a wave multiplies at a time: 16 * TILES outputs, 128 inputs, 16 rows.
template <int X, int TILES, int STEPS> struct Chunk {
    static constexpr int GROUPS = 4 / STEPS;
    u32x4 w[TILES];
    Eight<X> x[4];
    f32x4 s[GROUPS][TILES];
    uint32_t z[GROUPS][TILES];      // 16 bits: of a lane's four results; 8 bits: of its operand
    float xs[X == ROWS_I8 ? GROUPS : 1];
};

// A workgroup makes 16 * TILES outputs of 16 rows; its waves take every WAVES-th chunk of 128 inputs and add their sums in LDS.  Nothing is staged: a
// code is read once, straight from the image into the lane that multiplies it, DEPTH chunks ahead.  Lanes past the last row multiply it once
// more.  GROUPED: 8-bit rows with scales of groups.
// What bounds it: with few rows the memory (8 8-bit rows 4096 -> 32000 13.4 us for 71 MB, 5.3 TB/s) or, where the weights are small, the launch and one
// trip to memory (one bfloat16 row 9216 -> 4096 6.4 us, 20 MB); with more the rows' inputs, which every workgroup reads in pieces of 16 bytes.
template <int X, int TILES, int STEPS, bool GROUPED, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void w4_rows_kernel(W4Args a)
{
    typedef Form<X> F;
    typedef Chunk<X, TILES, STEPS> C;
    constexpr int GROUP = 32 * STEPS, XBYTES = X == ROWS_F32 ? 4 : X == ROWS_I8 ? 1 : 2, PITCH = 16 * TILES + 4;
    __shared__ __attribute__((aligned(16))) float red[WAVES][16][PITCH];
    const W4Layout l(a.out, a.in, GROUP);
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile0 = blockIdx.x * TILES, row0 = blockIdx.y * 16;
    // (a workgroup's tiles past the last one multiply the last once more)
    const u32x4 *codes[TILES];
    const float *scales[TILES];
    const uint8_t *zeros[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const size_t tile = min(tile0 + t, l.tiles - 1);
        codes[t] = reinterpret_cast<const u32x4 *>(a.image) + tile * l.chunks * 64 + lane;
        scales[t] = reinterpret_cast<const float *>(a.image + l.scale_at()) + tile * l.groups * 16 + 4 * quarter;
        zeros[t] = a.image + l.zero_at() + tile * l.groups * 16 + (X == ROWS_I8 ? col : 4 * quarter);
    }
    const size_t own_row = min(row0 + col, a.rows - 1);
    const char *xrow = static_cast<const char *>(a.x) + own_row * a.x_stride * XBYTES;
    const float *xscale = a.x_scale + own_row * a.x_groups;
    f32x4 total[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) total[t] = f32x4{0, 0, 0, 0};
    // whole: 128 inputs exist.  A group past the last input has sums of zero, whatever it is scaled with
    auto load = [&](C &c, int chunk, bool whole) {
#pragma unroll
        for (int t = 0; t < TILES; ++t) c.w[t] = codes[t][(size_t)chunk * 64];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = 128 * chunk + 32 * j + 8 * quarter;
            c.x[j].load(xrow, k, whole ? 8 : a.in - k);
        }
#pragma unroll
        for (int i = 0; i < C::GROUPS; ++i) {
            const int g = whole ? chunk * C::GROUPS + i : min(chunk * C::GROUPS + i, l.groups - 1);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                c.s[i][t] = *reinterpret_cast<const f32x4 *>(scales[t] + (size_t)g * 16);
                c.z[i][t] = X == ROWS_I8 ? zeros[t][(size_t)g * 16] : *reinterpret_cast<const uint32_t *>(zeros[t] + (size_t)g * 16);
            }
            if (GROUPED) c.xs[i] = xscale[g >> a.x_shift];
        }
    };
    auto multiply = [&](const C &c) {
        typename F::acc_t acc[TILES], sum;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j % STEPS == 0) {
                sum = typename F::acc_t{0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < TILES; ++t) acc[t] = typename F::acc_t{0, 0, 0, 0};
            }
            typename F::operand_t xo[F::PARTS];
            c.x[j].operands(xo);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                typename F::operand_t wide;
                if constexpr (X == ROWS_I8) wide = F::widen(c.w[t][j], c.z[j / STEPS][t] * 0x01010101u);
                else wide = F::widen(c.w[t][j]);
#pragma unroll
                for (int p = 0; p < F::PARTS; ++p) acc[t] = F::mfma(wide, xo[p], acc[t]);
            }
            if constexpr (X != ROWS_I8)
#pragma unroll
                for (int p = 0; p < F::PARTS; ++p) sum = F::mfma(F::ones(), xo[p], sum);
            if (j % STEPS != STEPS - 1) continue;
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float part;
                    if constexpr (X == ROWS_I8) part = GROUPED ? (float)acc[t][v] * c.xs[j / STEPS] : (float)acc[t][v];
                    else part = __builtin_fmaf(-(F::OFFSET + (float)(c.z[j / STEPS][t] >> (8 * v) & 255u)), sum[v], acc[t][v]);
                    total[t][v] = __builtin_fmaf(c.s[j / STEPS][t][v], part, total[t][v]);
                }
        }
    };
    const int whole = a.in / 128;
    C ring[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (wave + d * WAVES < whole) load(ring[d], wave + d * WAVES, true);
    for (int chunk = wave; chunk < whole; chunk += DEPTH * WAVES) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (chunk + d * WAVES >= whole) break;
            multiply(ring[d]);
            if (chunk + (d + DEPTH) * WAVES < whole) load(ring[d], chunk + (d + DEPTH) * WAVES, true);
        }
    }
    if (whole < l.chunks && wave == whole % WAVES) {        // the inputs past the last whole chunk
        load(ring[0], whole, false);
        multiply(ring[0]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) *reinterpret_cast<f32x4 *>(&red[wave][col][16 * t + 4 * quarter]) = total[t];
    __syncthreads();
    if (tid >= 64 * TILES) return;
    const int r = tid / (4 * TILES), q = tid % (4 * TILES), row = row0 + r, o = 16 * tile0 + 4 * q;
    if (row >= a.rows) return;
    f32x4 s = *reinterpret_cast<const f32x4 *>(&red[0][r][4 * q]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += *reinterpret_cast<const f32x4 *>(&red[w][r][4 * q]);
    if constexpr (X != ROWS_I8) s *= F::BACK;
    else if (!GROUPED) s *= a.x_scale[row];
    store_four(a.y, a.type, (size_t)row * a.out + o, s, a.out - o);
}

template <int X, bool GROUPED, int STEPS, int TILES, int DEPTH> void launch_rows(const W4Args &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.out + 16 * TILES - 1) / (16 * TILES)), (unsigned)((a.rows + 15) / 16));
    w4_rows_kernel<X, TILES, STEPS, GROUPED, 8, DEPTH><<<grid, dim3(512), 0, stream>>>(a);
}
// (chunks ahead: two of one or two tiles, but for float32 rows and groups of 32, which fill the registers.  Four of one tile 25.5 us for 8 8-bit rows
// 4096 -> 32000, two 24; sixteen waves 30)
template <int X, bool GROUPED, int STEPS> void launch_steps(const W4Args &a, int tiles, hipStream_t stream)
{
    constexpr int TWO = X == ROWS_F32 || STEPS == 1 ? 1 : 2;
    if (tiles == 4) launch_rows<X, GROUPED, STEPS, 4, 1>(a, stream);
    else if (tiles == 2) launch_rows<X, GROUPED, STEPS, 2, TWO>(a, stream);
    else launch_rows<X, GROUPED, STEPS, 1, TWO>(a, stream);
}
template <int X, bool GROUPED> xnor_status launch_groups(const W4Args &a, int group, int tiles, hipStream_t stream)
{
    if (group == 32) launch_steps<X, GROUPED, 1>(a, tiles, stream);
    else if (group == 64) launch_steps<X, GROUPED, 2>(a, tiles, stream);
    else launch_steps<X, GROUPED, 4>(a, tiles, stream);
    return hip_status(hipGetLastError());
}

}  // namespace

size_t w4_wimg_bytes(int out, int in, int group) { return W4Layout(out, in, group).bytes(); }

xnor_status launch_w4_quantize(const void *w, long long stride, uint8_t *codes, float *scale, uint8_t *zero, int out, int in, int group, int type,
                               hipStream_t stream)
{
    const int eights = (in + 31) / 32 * 4, threads = std::min(256, (eights + 63) / 64 * 64);
    by_type(type, [&](auto t) {
        w4_quantize_kernel<t()><<<dim3(std::min((unsigned)out, MOST_GROUPS)), dim3((unsigned)threads), 0, stream>>>(
            w, stride, reinterpret_cast<uint32_t *>(codes), scale, zero, out, in, group);
    });
    return hip_status(hipGetLastError());
}

xnor_status launch_w4_pack(const uint8_t *codes, const float *scale, const uint8_t *zero, void *wimg, int out, int in, int group, hipStream_t stream)
{
    const W4Layout l(out, in, group);
    const size_t items = l.scale_at() / 16 + (size_t)l.tiles * l.groups * 16;
    w4_pack_kernel<<<dim3((unsigned)std::min<size_t>((items + 255) / 256, MOST_GROUPS)), dim3(256), 0, stream>>>(
        reinterpret_cast<const uint32_t *>(codes), scale, zero, static_cast<uint8_t *>(wimg), out, in, group);
    return hip_status(hipGetLastError());
}

xnor_status launch_w4_linear(const void *x, long long x_stride, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group, int type,
                             hipStream_t stream)
{
    const W4Choice choice = w4_choice(rows, in, out, group, type);
    if (choice.kernel != W4_ROWS) return launch_w4_staged(choice.kernel, x, x_stride, nullptr, wimg, y, workspace, rows, in, out, group, 0, type, type, stream);
    const W4Args a{x, nullptr, static_cast<const uint8_t *>(wimg), y, x_stride, rows, in, out, 0, 0, type};
    if (type == XNOR_F32) return launch_groups<ROWS_F32, false>(a, group, choice.tiles, stream);
    if (type == XNOR_BF16) return launch_groups<ROWS_BF16, false>(a, group, choice.tiles, stream);
    return launch_groups<ROWS_F16, false>(a, group, choice.tiles, stream);
}

xnor_status launch_w4_linear_q8(const int8_t *q, const float *x_scale, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group,
                                int x_group, int type, hipStream_t stream)
{
    const W4Choice choice = w4_choice(rows, in, out, group, ROWS_I8);
    if (choice.kernel != W4_ROWS)
        return launch_w4_staged(choice.kernel, q, in, x_scale, wimg, y, workspace, rows, in, out, group, x_group, ROWS_I8, type, stream);
    const W4Args a{q, x_scale, static_cast<const uint8_t *>(wimg), y, in, rows, in, out, x_group ? (in + x_group - 1) / x_group : 0,
                   x_group ? __builtin_ctz(x_group / group) : 0, type};
    return x_group ? launch_groups<ROWS_I8, true>(a, group, choice.tiles, stream) : launch_groups<ROWS_I8, false>(a, group, choice.tiles, stream);
}

}  // namespace xnor
