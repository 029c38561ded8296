// Gradients of a product's weights and bias from the 8-bit rows that it read (contract: xnor_lowbit.h).
//
//     g_w[o][k] = sum_r g[r][o] x[r][k],    x = q * scale
// is a product of two matrices that both run along the rows, which neither stores next to each other.  Three launches:
//   range   the largest magnitude of every column of g (and its sum, the bias' gradient) and of the scales, in up to eight parts of the rows
//   stage   both matrices as float16 operands of the matrix instructions, transposed, each column multiplied by the power of two that brings its largest to between 2^14 and 2^15
//           (float16 then holds 8- and 11-bit gradients exactly down to 2^-28 of the largest, and less to 2^-39 of it)
//   product the sums, and the powers of two taken out again
// Few products go through none of it: gradient_direct_kernel below.
// With one scale per row the scale goes to g instead, sum_r (g[r][o] scale[r]) q[r][k], and q is an operand as it is: float32 gradients and weights then take two products of
// parts and not three (2048 rows 4096 -> 8192 472 and 277 us).
#include "xnor_internal.h"
#include "gradient_choice.h"
#include "lowbit.h"
#include "tiles.h"
#include <algorithm>
#include <cmath>

namespace xnor {

namespace {

constexpr int STAGED_COLS = 128;        // of a workgroup of the staging launch
constexpr int RANGE_COLS = 128, RANGE_PARTS = 8;        // of a workgroup of the first launch; of the rows, at most

// Where the launches keep what they hand on:
//   x, g     float16 [column][part][row], rows behind the last up to a whole 64 are 0
//   top, sum [part of the rows][columns]: largest magnitudes of g and of the scales, sums of g
//   e        exponents of the columns of g and of the groups
struct Places : GradientParts {
    int groups, parts, columns;
    size_t x_at, g_at, top_at, sum_at, e_at, total;
    __host__ __device__ Places(int rows, int in, int out, int group, int type, int w_type) : GradientParts(rows, group, type, w_type)
    {
        groups = group ? (in + group - 1) / group : 1;
        columns = (out + 3) / 4 * 4 + (groups + 3) / 4 * 4;     // (g's first, the groups from `groups_at` on)
        parts = (rows + 127) / 128 < RANGE_PARTS ? (rows + 127) / 128 : RANGE_PARTS;
        x_at = 0;
        g_at = x_at + (size_t)in * pitch_x();
        top_at = (g_at + (size_t)out * pitch_g() + 15) / 16 * 16;
        sum_at = top_at + (size_t)parts * columns * 4;
        e_at = sum_at + (size_t)parts * columns * 4;
        total = e_at + (size_t)columns * 4;
    }
    __host__ __device__ uint32_t pitch_x() const { return 2u * padded * parts_x; }
    __host__ __device__ uint32_t pitch_g() const { return 2u * padded * parts_g; }
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

// What stands for a column's largest: where its scales are the rows', the exponent of value times scale (as an exponent, since the product may be out of float32's range),
// otherwise the bits of the largest magnitude.  0: none that is finite and not 0.
constexpr uint32_t EXPONENT_0 = 4096;
__device__ __forceinline__ uint32_t size_of(float v)
{
    const uint32_t bits = __float_as_uint(v) & 0x7fffffffu;
    return bits < 0x7f800000u ? bits : 0u;
}
__device__ __forceinline__ uint32_t size_of(float v, float scale_mant, uint32_t scale_exp)
{
    const float m = __builtin_fabsf(__builtin_amdgcn_frexp_mantf(v) * scale_mant);         // (0.25 .. 1)
    const uint32_t e = (uint32_t)__builtin_amdgcn_frexp_expf(v) + scale_exp - (m < 0.5f ? 1 : 0);
    return m > 0.0f && m < __builtin_inff() ? e : 0u;
}

// Largest size and sum of a column: 16 lanes of 8 columns, 16 rows side by side in a workgroup of four waves, joined in LDS in one order.
// What bounds it: the memory (2048 x 8192 bfloat16 16 us alone, 34 MB).
template <int TYPE, bool BY_ROW> __device__ __forceinline__ void range_of(const GradArgs &a, const Places &p, const void *m, long long stride, int cols, int block, bool is_g)
{
    typedef real_t<TYPE> T;
    constexpr int WAVES = 4, AT_ONCE = 8;
    __shared__ uint32_t tops[WAVES][RANGE_COLS];
    __shared__ float sums[WAVES][RANGE_COLS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = RANGE_COLS * block + 8 * (lane & 15), n = cols - c;
    const int first = (int)((long long)a.rows * blockIdx.y / p.parts), last = (int)((long long)a.rows * (blockIdx.y + 1) / p.parts);
    uint32_t t[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    auto take = [&](const Real8<TYPE> &v, float scale) {
        const float mant = __builtin_amdgcn_frexp_mantf(scale);
        const uint32_t exp = EXPONENT_0 + __builtin_amdgcn_frexp_expf(scale);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t[j] = max(t[j], BY_ROW ? size_of(v[j], mant, exp) : size_of(v[j]));
            s[j] += v[j];
        }
    };
    const T *from = static_cast<const T *>(m) + c;
    int r = first + 4 * wave + (lane >> 4);
    if (n >= 8)
        for (; r + 4 * WAVES * (AT_ONCE - 1) < last; r += 4 * WAVES * AT_ONCE) {
            Real8<TYPE> v[AT_ONCE];
            float scale[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                v[i].load(from + (size_t)(r + 4 * WAVES * i) * stride, 8);
                scale[i] = BY_ROW ? a.scale[r + 4 * WAVES * i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) take(v[i], scale[i]);
        }
    for (; r < last; r += 4 * WAVES) {
        Real8<TYPE> v;
        v.load(from + (size_t)r * stride, n);
        take(v, BY_ROW ? a.scale[r] : 0.0f);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int d = 16; d < 64; d <<= 1) {
            t[j] = max(t[j], (uint32_t)__shfl_xor((int)t[j], d, 64));
            s[j] += __shfl_xor(s[j], d, 64);
        }
        if (lane < 16) {
            tops[wave][8 * lane + j] = t[j];
            sums[wave][8 * lane + j] = s[j];
        }
    }
    __syncthreads();
    const int i = threadIdx.x, o = RANGE_COLS * block + i;
    if (i >= RANGE_COLS || o >= cols) return;
    uint32_t top = 0;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        top = max(top, tops[w][i]);
        sum += sums[w][i];
    }
    const int at = is_g ? o : p.groups_at(a.out) + o;
    reinterpret_cast<uint32_t *>(a.work + p.top_at)[(size_t)blockIdx.y * p.columns + at] = top;
    if (is_g) reinterpret_cast<float *>(a.work + p.sum_at)[(size_t)blockIdx.y * p.columns + at] = sum;
}

template <int TYPE> __global__ __launch_bounds__(256) void gradient_range_kernel(GradArgs a)
{
    const Places p(a.rows, a.in, a.out, a.group, a.type, a.w_type);
    const int blocks_g = (a.out + RANGE_COLS - 1) / RANGE_COLS;
    if ((int)blockIdx.x >= blocks_g) range_of<XNOR_F32, false>(a, p, a.scale, p.groups, p.groups, blockIdx.x - blocks_g, false);      // (not with scales of rows)
    else if (p.by_row) range_of<TYPE, true>(a, p, a.g, a.g_stride, a.out, blockIdx.x, true);
    else range_of<TYPE, false>(a, p, a.g, a.g_stride, a.out, blockIdx.x, true);
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
        if (is_g || !p.by_row)
#pragma unroll
            for (int i = 0; i < RANGE_PARTS; ++i) most = max(most, top[(size_t)min(i, p.parts - 1) * p.columns]);
        int e;
        if (p.by_row) e = !is_g ? 0 : most ? (int)(most - EXPONENT_0) - 15 : 0;
        else e = __builtin_amdgcn_frexp_expf(__uint_as_float(most)) - (is_g ? 15 : 8);       // (an 8-bit number brings 2^7)
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
            const float scale = p.by_row && n > 0 ? a.scale[r0 + r] : 1.0f, mant = __builtin_amdgcn_frexp_mantf(scale);
            const int exp = __builtin_amdgcn_frexp_expf(scale);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                to[j] = j >= n ? 0.0f : __builtin_amdgcn_ldexpf(__builtin_amdgcn_frexp_mantf(v[j]) * mant, __builtin_amdgcn_frexp_expf(v[j]) + exp - exponents[c + j]);
        } else {
            Eight<ROWS_I8> v;
            v.load(a.q + (size_t)(r0 + r) * a.in + c0, c, n);
            const float s = p.by_row ? 1.0f : n > 0 ? a.scale[(size_t)(r0 + r) * p.groups + (c0 + c) / a.group] : 0.0f;
            const float scaled = n > 0 ? __builtin_amdgcn_ldexpf(s, -exponents[c]) : 0.0f;       // (eight columns are of one group)
#pragma unroll
            for (int j = 0; j < 8; ++j) to[j] = j < n ? (float)(int8_t)(v.w[j / 4] >> (8 * (j & 3))) * scaled : 0.0f;
        }
    }
    __syncthreads();
    // eight lanes write the 64 rows of a column.  (One unit at a time: side by side, which is no faster, the last stores end the program without an instruction behind them, and a
    // reader of the listing takes the next program's first ones for what overwrites their registers.)
    const int parts = is_g ? p.parts_g : p.parts_x;
    uint8_t *to = a.work + (is_g ? p.g_at : p.x_at);
#pragma unroll 1
    for (int i = 0; i < STAGED_COLS * STAGED_ROWS / 8 / 256; ++i) {
        const int unit = tid + 256 * i, col = unit >> 3, r = 8 * (unit & 7);
        if (c0 + col >= cols) break;
        const float *from = tile + r * PITCH + col;
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = from[j * PITCH];
            hi[j] = (_Float16)v;
            const float rest = v - (float)hi[j];
            lo[j] = (_Float16)(__builtin_fabsf(v) < __builtin_inff() ? rest : 0.0f);
        }
        uint8_t *at = to + ((size_t)(c0 + col) * parts * p.padded + r0 + r) * 2;
        *reinterpret_cast<u32x4 *>(at) = __builtin_bit_cast(u32x4, hi);
        if (parts == 2) *reinterpret_cast<u32x4 *>(at + 2 * (size_t)p.padded) = __builtin_bit_cast(u32x4, lo);
    }
}

// Four neighbouring results, `n` of which exist, to g_w[at], or added to what is there.
__device__ __forceinline__ void add_results(const GradArgs &a, size_t at, f32x4 v, int n)
{
    if (a.accumulate)
#pragma unroll
        for (int m = 0; m < 4; ++m)
            if (m < n)
                v[m] += a.w_type == XNOR_F32    ? static_cast<const float *>(a.g_w)[at + m]
                        : a.w_type == XNOR_BF16 ? (float)static_cast<const __bf16 *>(a.g_w)[at + m]
                                                : (float)static_cast<const _Float16 *>(a.g_w)[at + m];
    store_four(a.g_w, a.w_type, at, v, n);
}

constexpr int TURNED = 32 * (64 * 4 + 16);          // bytes of 32 outputs x 64 inputs, outputs 16 bytes further apart
template <class P> constexpr int lds_bytes() { return std::max(P::BUFFERS * P::BYTES, P::WAVES * TURNED); }

// What bounds it: 2048 rows 4096 -> 8192, bfloat16 throughout, 134 to 140 us by itself (a library's product of bfloat16 matrices of these sizes 116): matrix instructions and the
// loads of their operands, which overlap in part; the range takes 17 and the staging 28 (88 MB), all three one behind the other 164 to 176.  256 rows 9216 -> 4096 to float32 58 us: 32 with
// the first chunk alone (151 MB of results), 4 more for each of the other seven (57 MB out of L2), which the results hardly hide (tiles of 256 x 128, more of them in LDS or on a CU,
// waves of two priorities, stores past the caches or without turning: 3 us at most).
template <class P> __global__ __launch_bounds__(64 * P::WAVES) void gradient_product_kernel(GradArgs a, int blocks_x, int blocks_g)
{
    constexpr int WA = P::WA, TA = P::TA, TB = P::TB, WIDE = TA % 2 ? 1 : 2, PER_ROW = 8 * WIDE;           // tiles of a turn; 16-byte pieces of an output in it
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Places p(a.rows, a.in, a.out, a.group, a.type, a.w_type);
    int bx, bg;
    if (!tile_of(blocks_x, blocks_g, bx, bg)) return;
    f32x16 acc[TA][TB];
    const Side x{a.work + p.x_at, p.pitch_x(), a.in, 2u * p.padded}, g{a.work + p.g_at, p.pitch_g(), a.out, 2u * p.padded};
    tile_product<HalfOp, P, true, true>(acc, lds, x, g, bx * P::A, bg * P::B, 0, 2 * p.padded / P::KB, 2 * p.padded);
    // A wave turns 32 outputs x 64 (32) inputs in LDS, so that an output's are stored next to each other.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wx = wave % WA, wg = wave / WA;
    uint8_t *turned = lds + wave * TURNED;
    const int *e = reinterpret_cast<const int *>(a.work + p.e_at);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int o0 = bg * P::B + (wg * TB + j) * 32, eg = e[min(o0 + (lane & 31), a.out - 1)];
#pragma unroll
        for (int pair = 0; pair < TA; pair += WIDE) {
            const int k0 = bx * P::A + (wx * TA + pair) * 32;
#pragma unroll
            for (int i = pair; i < pair + WIDE; ++i) {
                const int k = k0 + (i - pair) * 32, ex = e[p.groups_at(a.out) + (a.group ? min(k, a.in - 1) / a.group : 0)] + eg;     // (groups are whole tiles)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    f32x4 v;
#pragma unroll
                    for (int m = 0; m < 4; ++m) v[m] = __builtin_amdgcn_ldexpf(acc[i][j][4 * b + m], ex);
                    *reinterpret_cast<f32x4 *>(turned + (lane & 31) * (64 * 4 + 16) + 4 * ((i - pair) * 32 + 8 * b + 4 * (lane >> 5))) = v;
                }
            }
            // (a wave's own place: its lanes run in step, and what it writes there it reads itself)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int n = 0; n < PER_ROW / 2; ++n) {
                const int r = 64 / PER_ROW * n + lane / PER_ROW, k = 4 * (lane % PER_ROW), left = a.in - k0 - k;
                if (o0 + r >= a.out || left <= 0) continue;
                f32x4 v = *reinterpret_cast<const f32x4 *>(turned + r * (64 * 4 + 16) + 4 * k);
                const size_t at = (size_t)(o0 + r) * a.in + k0 + k;
                add_results(a, at, v, left);
            }
            asm volatile("" ::: "memory");
        }
    }
}

// Few products: one launch, 64 outputs x 64 inputs to a workgroup, in float32 throughout.  The matrix instructions of two rows take their operands as they lie: a lane's are one row's,
// neighbouring lanes' neighbouring columns (two of them each, for two tiles).  Eight waves share the rows, two at a time, and their sums meet in LDS.
// What bounds it: launch, first loads and last sums up to 64 rows (6.4 us), behind them 0.022 us a row for up to 256 workgroups, 1.6 times what the matrix instructions take
// at 2.4 GHz (addresses by steps in place of products, more rows ahead: no change).
constexpr int DIRECT_WAVES = 8;
struct DirectShared {
    f32x4 sums[DIRECT_WAVES][2][2][4][64];          // [wave][input of a pair][output of a pair][register / 4][lane]
    float bias[DIRECT_WAVES][DIRECT_SIDE];
};

template <int TYPE> __global__ __launch_bounds__(64 * DIRECT_WAVES) void gradient_direct_kernel(GradArgs a, int blocks_x)
{
    typedef real_t<TYPE> T;
    constexpr int AT_ONCE = 4;
    struct __attribute__((packed, aligned(sizeof(T)))) Pair { T v[2]; };
    struct __attribute__((packed)) Codes { int8_t v[2]; };
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    DirectShared &s = *reinterpret_cast<DirectShared *>(lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pair = 2 * (lane & 31);
    const int bo = blockIdx.x / blocks_x, c0 = DIRECT_SIDE * (int)(blockIdx.x - bo * blocks_x), o0 = DIRECT_SIDE * bo;
    const int groups = a.group ? (a.in + a.group - 1) / a.group : 1;
    // the last column of an odd number comes as the second of the pair before; columns behind the last are somebody's results that are not kept
    const int c = c0 + pair, o = o0 + pair, c_at = min(c, a.in - 2), o_at = min(o, a.out - 2), group = a.group ? min(c, a.in - 1) / a.group : 0;
    const int8_t *q = a.q + c_at;
    const float *scale = a.scale + group;
    const T *g = static_cast<const T *>(a.g) + o_at;
    struct Step {
        Codes q;
        Pair g;
        float scale;
    };
    auto load = [&](Step &t, int r) {
        const size_t row = min(r, a.rows - 1);
        t.q = *reinterpret_cast<const Codes *>(q + row * a.in);
        t.scale = scale[row * groups];
        t.g = *reinterpret_cast<const Pair *>(g + row * a.g_stride);
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[i >> 1][i & 1][k] = 0.0f;
    float bias[2] = {0.0f, 0.0f};
    Step next[AT_ONCE];
    const int own = 2 * wave + (lane >> 5);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) load(next[i], own + 2 * DIRECT_WAVES * i);
    for (int r = own; r - (lane >> 5) < a.rows; r += 2 * DIRECT_WAVES * AT_ONCE) {            // (a wave's lanes end together)
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const Step t = next[i];
            load(next[i], r + 2 * DIRECT_WAVES * (i + AT_ONCE));
            asm volatile("" ::: "memory");              // (else the loads wait until they are used: 777 rows 26 us, so 25)
            const bool is = r + 2 * DIRECT_WAVES * i < a.rows;
            float x[2], y[2];
            auto rows_of = [&](float scale) {
                x[1] = is ? (float)t.q.v[1] * scale : 0.0f;
                x[0] = c > c_at ? x[1] : is ? (float)t.q.v[0] * scale : 0.0f;
            };
            auto multiply = [&]() {
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[k >> 1][k & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[k >> 1], y[k & 1], acc[k >> 1][k & 1], 0, 0, 0);
            };
            y[1] = is ? (float)t.g.v[1] : 0.0f;
            y[0] = o > o_at ? y[1] : is ? (float)t.g.v[0] : 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k) bias[k] += y[k];
            // 127 times a scale of 2^121 and more is out of range where its product with a small gradient is not: such scales' part of 2^8 goes to the gradients, in
            // instructions of their own.  (Gradients of 2^120 and more stay the largest number there: with any code but 0 that is an infinity all the same.)  To ask
            // takes 0.3 to 0.7 us of 11 to 14 with 16-bit gradients (256 rows 1024 -> 1024, 400 rows 512 -> 512), nothing with float32.
            const float size = __builtin_fabsf(t.scale);
            const bool large = size >= 0x1p120f && size < __builtin_inff();
            rows_of(large ? 0.0f : t.scale);
            multiply();
            if (__any(large)) {
                rows_of(large ? t.scale * 0x1p-8f : 0.0f);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    y[k] = __builtin_fabsf(y[k]) < __builtin_inff() ? __builtin_fminf(__builtin_fmaxf(y[k] * 0x1p8f, -0x1.fffffep127f), 0x1.fffffep127f) : y[k];
                multiply();
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            f32x4 v;
#pragma unroll
            for (int m = 0; m < 4; ++m) v[m] = acc[k >> 1][k & 1][4 * b + m];
            s.sums[wave][k >> 1][k & 1][b][lane] = v;
        }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float both = bias[k] + __shfl_xor(bias[k], 32, 64);
        if (lane < 32) s.bias[wave][pair + k] = both;
    }
    __syncthreads();
    // a thread: eight neighbouring inputs of an output
    const int b = wave & 3, j = wave >> 2, row = o0 + pair + j, first = c0 + 16 * b + 8 * (lane >> 5);
    f32x4 even = s.sums[0][0][j][b][lane], odd = s.sums[0][1][j][b][lane];
#pragma unroll
    for (int w = 1; w < DIRECT_WAVES; ++w) {
        even += s.sums[w][0][j][b][lane];
        odd += s.sums[w][1][j][b][lane];
    }
    if (row < a.out)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int k = first + 4 * half, left = a.in - k;
            if (left <= 0) break;
            f32x4 v = {even[2 * half], odd[2 * half], even[2 * half + 1], odd[2 * half + 1]};
            add_results(a, (size_t)row * a.in + k, v, left);
        }
    if (a.g_bias && c0 == 0 && threadIdx.x < DIRECT_SIDE && o0 + (int)threadIdx.x < a.out) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < DIRECT_WAVES; ++w) sum += s.bias[w][threadIdx.x];
        float &to = a.g_bias[o0 + threadIdx.x];
        to = a.accumulate ? to + sum : sum;
    }
}

template <class P> xnor_status launch_plan(const GradArgs &a, hipStream_t stream)
{
    constexpr unsigned lds = lds_bytes<P>();
    const int blocks_x = (a.in + P::A - 1) / P::A, blocks_g = (a.out + P::B - 1) / P::B;
    const long long count = (long long)blocks_x * blocks_g;             // (2^23 and some where they are smallest, with 256 threads each)
    auto kernel = gradient_product_kernel<P>;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return XNOR_ERR_HIP;
    kernel<<<dim3((unsigned)((count + 7) / 8 * 8)), dim3(64 * P::WAVES), lds, stream>>>(a, blocks_x, blocks_g);
    return hip_status(hipGetLastError());
}

xnor_status launch_product(const GradArgs &a, const Places &p, int side, hipStream_t stream)
{
    if (p.parts_x == 1 && p.parts_g == 2) {
        if (side == 256) return launch_plan<TilePlan<2, 4, 4, 2, 64, 3, 1, 2>>(a, stream);
        return side == 128 ? launch_plan<TilePlan<2, 4, 2, 1, 64, 3, 1, 2>>(a, stream) : launch_plan<TilePlan<2, 2, 1, 1, 128, 4, 1, 2>>(a, stream);
    }
    if (p.parts_x == 1) {
        if (side == 256) return launch_plan<TilePlan<2, 4, 4, 2, 128, 2>>(a, stream);
        return side == 128 ? launch_plan<TilePlan<2, 4, 2, 1, 128, 2>>(a, stream) : launch_plan<TilePlan<2, 2, 1, 1, 128, 4>>(a, stream);
    }
    if (p.parts_g == 1) {
        if (side == 256) return launch_plan<TilePlan<2, 4, 4, 2, 64, 3, 2, 1>>(a, stream);
        return side == 128 ? launch_plan<TilePlan<2, 4, 2, 1, 64, 3, 2, 1>>(a, stream) : launch_plan<TilePlan<2, 2, 1, 1, 128, 4, 2, 1>>(a, stream);
    }
    return side == 128 ? launch_plan<TilePlan<2, 4, 2, 1, 64, 2, 2, 2>>(a, stream) : launch_plan<TilePlan<2, 2, 1, 1, 128, 3, 2, 2>>(a, stream);
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
    const GradientChoice choice = gradient_choice(p, rows, in, out, (int)type_bytes(w_type));
    xnor_status status = XNOR_OK;
    if (choice.direct) {
        const int blocks_x = (in + DIRECT_SIDE - 1) / DIRECT_SIDE, blocks_g = (out + DIRECT_SIDE - 1) / DIRECT_SIDE;
        by_type(type, [&](auto t) {
            auto kernel = gradient_direct_kernel<t()>;
            if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(DirectShared)) != hipSuccess) {
                status = XNOR_ERR_HIP;
                return;
            }
            kernel<<<dim3((unsigned)(blocks_x * blocks_g)), dim3(64 * DIRECT_WAVES), sizeof(DirectShared), stream>>>(a, blocks_x);
            status = hip_status(hipGetLastError());
        });
        return status;
    }
    const int scale_blocks = p.by_row ? 0 : (p.groups + RANGE_COLS - 1) / RANGE_COLS;
    const dim3 range((unsigned)((out + RANGE_COLS - 1) / RANGE_COLS + scale_blocks), (unsigned)p.parts);
    const dim3 stage((unsigned)((out + STAGED_COLS - 1) / STAGED_COLS + (in + STAGED_COLS - 1) / STAGED_COLS), (unsigned)(p.padded / STAGED_ROWS));
    by_type(type, [&](auto t) {
        gradient_range_kernel<t()><<<range, dim3(256), 0, stream>>>(a);
        status = hip_status(hipGetLastError());
        if (status) return;
        gradient_stage_kernel<t()><<<stage, dim3(256), 0, stream>>>(a);
        status = hip_status(hipGetLastError());
    });
    if (status) return status;
    return launch_product(a, p, choice.side, stream);
}

}  // namespace xnor
