// Rows to 8 bits, activation functions that keep their input in 8 bits, and their backward pass (contracts: xnor_lowbit.h).
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr float TINY = 0x1p-100f;           // groups whose largest magnitude is below hold zeros

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }     // (orders like |v|, infinities and NaN last)

// The largest over the threads of a row (blockDim.x, whole waves); `slots` holds a word per wave of the row and is not used again before a barrier.
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *slots)
{
    v = wave_max(v);
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slots[wave] = v;
    __syncthreads();
    for (int i = 0; i < waves; ++i) v = max(v, slots[i]);
    return v;
}
// The largest of the group of columns that a lane's eight belong to: a group is 4, 8 or 16 neighbouring lanes.
__device__ __forceinline__ uint32_t group_max(uint32_t v, int group)
{
    for (int s = group / 16; s > 0; s >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, s, 64));
    return v;
}

// Eight columns from c on in 8 bits, under the largest magnitude of their row or group.
__device__ __forceinline__ void to_8_bits(const float *v, uint32_t top, int8_t *q, float *scale, size_t row, int c, int cols, int group)
{
    const int n = cols - c;
    if (n <= 0) return;
    const float largest = __uint_as_float(top);
    const bool finite = top < 0x7f800000u, some = largest >= TINY;
    const float factor = finite && some ? 127.0f / largest : 0.0f;
    union {
        int8_t b[8];
        uint32_t w[2];
    } r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.b[j] = (int8_t)(int)(finite ? __builtin_rintf(v[j] * factor) : 0.0f);
    const float s = !finite ? __builtin_nanf("") : some ? largest / 127.0f : 0.0f;
    if (group == 0 ? c == 0 : (c & (group - 1)) == 0) scale[group == 0 ? row : row * ((cols + group - 1) / group) + c / group] = s;
    int8_t *p = q + row * cols + c;
    if (n >= 8) {
        typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(1)));
        *reinterpret_cast<words2 *>(p) = words2{r.w[0], r.w[1]};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = r.b[j];
    }
}

// The root of e^(-a) for a = hi + lo >= 0, to about 1.5 units in the last place: the instruction has no results below the normal numbers, products of two roots do.
// Its base-2 exponent is in two numbers, the second to first order.  (expf spends twice as much on ranges.)
__device__ __forceinline__ float root_exp_minus(float hi, float lo)
{
    constexpr float log2e = 0.721347520f, rest = 9.62981495e-9f;        // halved
    const float t = hi * -log2e, err = __builtin_fmaf(hi, -log2e, -t) - __builtin_fmaf(lo, log2e, hi * rest);
    const float e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, err * 0.693147181f, e);
}
// 1 / d for 1 <= d, one step of Newton's iteration behind the instruction's
__device__ __forceinline__ float reciprocal(float d)
{
    const float r = __builtin_amdgcn_rcpf(d);
    return __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
}
// |x|, no farther out than where e^(-|x| / 2) is 0: times that an infinity would be NaN; a NaN stays one
__device__ __forceinline__ float near_zero(float x)
{
    const float a = __builtin_fabsf(x);
    return a > 1e4f ? 1e4f : a;
}

// f(x) and f'(x) from e^-|x| or e^(-x^2 / 2), which never overflow; a NaN stays one.
template <int F> struct Point {
    float value, slope;
    __device__ __forceinline__ explicit Point(float x)
    {
        if (F == XNOR_RELU) {
            value = x > 0.0f ? x : x != x ? x : 0.0f;
            slope = x > 0.0f ? 1.0f : x != x ? x : 0.0f;
        } else if (F == XNOR_GELU) {
            // Phi(-|x|) = erfc(z) / 2 with z = |x| / sqrt 2;  erfc(z) e^(z^2) / t is nearly a polynomial of t = 1 / (1 + z / 2) (the substitution of Press et al., Numerical
            // Recipes, sec. 6.2).  These coefficients are a fit to its values in 64 bits, made here, and are within 8.4e-8 of it up to |x| = 14.5, where the results end; what
            // comes out is within 5.2e-7 of GELU(x) down to x = -12.  (erfcf takes three times as long.)
            const float a = near_zero(x), square = a * a, root = root_exp_minus(0.5f * square, 0.5f * __builtin_fmaf(a, a, -square));
            const float t = reciprocal(__builtin_fmaf(a, 0.353553391f, 1.0f));
            constexpr float c[9] = {0.2820855975f, 0.2823898494f, 0.2429982424f, 0.2031030208f, -0.02760601416f, 0.2794856131f, -0.4884357750f, 0.2851699591f, -0.05919053033f};
            float q = c[8];
#pragma unroll
            for (int i = 7; i >= 0; --i) q = __builtin_fmaf(q, t, c[i]);
            const float part = 0.5f * root * (t * q), tail = part * root, out = a * root;
            value = __builtin_fmaf(-out, part, __builtin_fmaxf(x, 0.0f));
            slope = __builtin_fmaf(__builtin_copysignf(out, x), 0.398942280f * root, x >= 0.0f ? 1.0f - tail : tail);
        } else {
            const float a = near_zero(x), root = root_exp_minus(a, 0.0f), e = root * root, r = reciprocal(1.0f + e);
            const float out = a * root, part = root * r;                         // |x| e^(-|x| / 2) and what makes it |x| / (1 + e^|x|)
            value = x >= 0.0f ? x * r : -out * part;
            slope = x >= 0.0f ? __builtin_fmaf(out * part, r, r) : __builtin_fmaf(-out * part, r, e * r);
        }
    }
};
template <int F> __device__ __forceinline__ float value_of(float x) { return Point<F>(x).value; }

struct RowArgs {
    const void *x;
    void *y;
    int8_t *q, *kept;
    float *scale, *kept_scale;
    long long x_stride;
    int rows, cols, group, kept_group;
};

// A row per workgroup (blockDim.y rows of one wave each where they are narrow).  STEPS > 0: thread t holds the eight columns from 8 * (t + i * threads) on, i < STEPS;
// STEPS = 0: rows of any width, read again once their largest is known.
// What bounds it: the memory, with the wait for the largest between a row's reads and writes (2048 x 4096 bfloat16 8.8 us, 2.9 TB/s; 2048 x 9216 13.8 us, 4.1 TB/s), and the
// launch below some hundred rows (7.6 us from call to call).
template <int TYPE, int STEPS> __global__ __launch_bounds__(1024) void q8_rows_kernel(RowArgs a)
{
    typedef real_t<TYPE> T;
    __shared__ uint32_t slots[16];
    const int row = blockIdx.x * blockDim.y + threadIdx.y, tid = threadIdx.x, step = 8 * blockDim.x;
    if (row >= a.rows) return;                  // (whole waves; side by side only where no barrier follows)
    const T *x = static_cast<const T *>(a.x) + (size_t)row * a.x_stride;
    if constexpr (STEPS > 0) {
        Real8<TYPE> v[STEPS];
        uint32_t top[STEPS], all = 0;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) v[i].load(x + 8 * tid + i * step, a.cols - 8 * tid - i * step);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            top[i] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top[i] = max(top[i], magnitude(v[i][j]));
            all = max(all, top[i]);
        }
        if (a.group == 0) all = row_max(all, slots);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = v[i][j];
            to_8_bits(f, a.group ? group_max(top[i], a.group) : all, a.q, a.scale, row, 8 * tid + i * step, a.cols, a.group);
        }
    } else {
        uint32_t all = 0;
        if (a.group == 0) {
            for (int c = 8 * tid; c < a.cols; c += step) {
                Real8<TYPE> v;
                v.load(x + c, a.cols - c);
#pragma unroll
                for (int j = 0; j < 8; ++j) all = max(all, magnitude(v[j]));
            }
            all = row_max(all, slots);
        }
        for (int c0 = 0; c0 < a.cols; c0 += step) {            // (all lanes: groups exchange their largest)
            const int c = c0 + 8 * tid;
            Real8<TYPE> v;
            v.load(x + c, a.cols - c);
            float f[8];
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[j] = v[j];
                top = max(top, magnitude(f[j]));
            }
            to_8_bits(f, a.group ? group_max(top, a.group) : all, a.q, a.scale, row, c, a.cols, a.group);
        }
    }
}

// Eight columns' values of f (times the other half's), and what they were made from.
template <int TYPE, int F, bool GATED> struct Act8 {
    float x[8], up[8], a[8];
    __device__ __forceinline__ void make(const Real8<TYPE> &v, const Real8<TYPE> &u)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = v[j];
            a[j] = value_of<F>(x[j]);
            if (GATED) {
                up[j] = u[j];
                a[j] *= up[j];
            }
        }
    }
    __device__ __forceinline__ static uint32_t top(const float *f)
    {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) t = max(t, magnitude(f[j]));
        return t;
    }
};

// The same rows through f.  kept only where the halves of a gated row are whole groups (and eights) of columns: otherwise q8_rows_kernel writes it.
// What bounds it: the vector unit, and the memory behind it: 2048 x 4096 bfloat16, values and kept: GELU 16 us, of which vector instructions take 13 (19.5 us with erfcf and
// expf); SiLU of gated rows 19 us, 15 of them (67 MB at the copy's rate 13.5).  ReLU of 2048 x 9216 waits for the memory: 21.5 us, 94 MB at 4.4 TB/s.  Gated rows whose halves are not whole groups go through both kernels: 25.7 us for 2048 x 4100.
template <int TYPE, int F, bool GATED, int STEPS> __global__ __launch_bounds__(1024) void activation_kernel(RowArgs a)
{
    typedef real_t<TYPE> T;
    typedef Act8<TYPE, F, GATED> A;
    __shared__ uint32_t slots[2][16];
    const int row = blockIdx.x * blockDim.y + threadIdx.y, tid = threadIdx.x, step = 8 * blockDim.x;
    if (row >= a.rows) return;
    const int wide = GATED ? 2 * a.cols : a.cols;
    const T *x = static_cast<const T *>(a.x) + (size_t)row * a.x_stride;
    T *y = static_cast<T *>(a.y) + (size_t)row * a.cols;
    const bool all_q = a.q && a.group == 0, all_kept = a.kept && a.kept_group == 0;
    uint32_t top = 0, kept_top = 0;
    auto write = [&](const A &v, int c) {
        const int n = a.cols - c;
        if (a.y) {
            Real8<TYPE> o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o.v[j] = (T)v.a[j];
            o.store(y + c, n);
        }
        if (a.q) to_8_bits(v.a, a.group ? group_max(A::top(v.a), a.group) : top, a.q, a.scale, row, c, a.cols, a.group);
        if (a.kept) {
            const uint32_t own = a.kept_group ? group_max(A::top(v.x), a.kept_group) : kept_top;
            if (GATED) {            // (columns past the first half are the other's)
                if (n > 0) to_8_bits(v.x, own, a.kept, a.kept_scale, row, c, wide, a.kept_group);
                const uint32_t other = a.kept_group ? group_max(A::top(v.up), a.kept_group) : kept_top;
                if (n > 0) to_8_bits(v.up, other, a.kept, a.kept_scale, row, a.cols + c, wide, a.kept_group);
            } else {
                to_8_bits(v.x, own, a.kept, a.kept_scale, row, c, a.cols, a.kept_group);
            }
        }
    };
    auto load = [&](Real8<TYPE> &v, Real8<TYPE> &u, int c) {
        v.load(x + c, a.cols - c);
        if (GATED) u.load(x + a.cols + c, a.cols - c);
    };
    auto largest = [&]() {
        if (all_q) top = row_max(top, slots[0]);
        if (all_kept) kept_top = row_max(kept_top, slots[1]);
    };
    if constexpr (STEPS > 0) {
        Real8<TYPE> v[STEPS], u[STEPS];
        A f[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) load(v[i], u[i], 8 * tid + i * step);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            f[i].make(v[i], u[i]);
            if (all_q) top = max(top, A::top(f[i].a));
            if (all_kept) kept_top = max(kept_top, max(A::top(f[i].x), GATED ? A::top(f[i].up) : 0u));
        }
        largest();
#pragma unroll
        for (int i = 0; i < STEPS; ++i) write(f[i], 8 * tid + i * step);
    } else {
        if (all_q || all_kept)
            for (int c = 8 * tid; c < a.cols; c += step) {
                Real8<TYPE> v, u;
                A f;
                load(v, u, c);
                f.make(v, u);
                top = max(top, A::top(f.a));
                kept_top = max(kept_top, max(A::top(f.x), GATED ? A::top(f.up) : 0u));
            }
        largest();
        for (int c0 = 0; c0 < a.cols; c0 += step) {
            Real8<TYPE> v, u;
            A f;
            load(v, u, c0 + 8 * tid);
            f.make(v, u);
            write(f, c0 + 8 * tid);
        }
    }
}

struct BackwardArgs {
    const int8_t *kept;
    const float *kept_scale;
    const void *g;
    void *g_x;
    long long g_stride;
    int rows, cols, shift, groups, per_row;             // shift: of a column to its group (31: one for the row); groups: of a kept row; per_row: workgroups beside each other
};

// Eight neighbours of kept, widened; n: how many exist.
__device__ __forceinline__ void kept_8(const int8_t *p, int n, float *v)
{
    uint32_t w[2] = {0, 0};
    if (n >= 8) {
        typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(1)));
        const words2 t = *reinterpret_cast<const words2 *>(p);
        w[0] = t.x;
        w[1] = t.y;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) w[j / 4] |= (uint32_t)(uint8_t)p[j] << (8 * (j & 3));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(w[j / 4] >> (8 * (j & 3)));
}

// Eight columns per thread, blockDim.y rows per workgroup, so that rows and columns take no division per thread and scales none per value (both together 23.8 us instead of
// 19.4 below).  What bounds it: 2048 x 4096 bfloat16, GELU 15.5 us, of which vector instructions take 11 (42 MB at the copy's rate 8.5); SiLU of gated rows 19.5 us, 67 MB
// (13.5) beside 10 of vector instructions, four streams of rows at once; ReLU of 2048 x 9216 the memory, 17 to 20 us, 4.7 TB/s and more.
template <int TYPE, int F, bool GATED> __global__ __launch_bounds__(256) void activation_grad_kernel(BackwardArgs a)
{
    typedef real_t<TYPE> T;
    const int set = (int)(blockIdx.x / a.per_row), row = set * blockDim.y + threadIdx.y;
    const int c = 8 * (int)((blockIdx.x - set * a.per_row) * blockDim.x + threadIdx.x), n = a.cols - c;
    if (row >= a.rows || n <= 0) return;
    const int wide = GATED ? 2 * a.cols : a.cols;
    const int8_t *kept = a.kept + (size_t)row * wide;
    const float *scale = a.kept_scale + (size_t)row * a.groups;
    Real8<TYPE> g, o;
    g.load(static_cast<const T *>(a.g) + (size_t)row * a.g_stride + c, n);
    T *g_x = static_cast<T *>(a.g_x) + (size_t)row * wide;
    float x[8];
    kept_8(kept + c, n, x);
    const float s = scale[c >> a.shift];
    if (GATED) {
        float up[8], su[8];
        kept_8(kept + a.cols + c, n, up);
        if (a.cols % 8 == 0) {
            const float all = scale[(a.cols + c) >> a.shift];           // (eights of the other half are of one group too)
#pragma unroll
            for (int j = 0; j < 8; ++j) su[j] = all;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) su[j] = scale[min(a.cols + c + j, wide - 1) >> a.shift];
        }
        Real8<TYPE> other;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const Point<F> p(x[j] * s);
            o.v[j] = (T)(g[j] * (up[j] * su[j]) * p.slope);
            other.v[j] = (T)(g[j] * p.value);
        }
        o.store(g_x + c, n);
        other.store(g_x + a.cols + c, n);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = (T)(g[j] * Point<F>(x[j] * s).slope);
        o.store(g_x + c, n);
    }
}

// Threads of a row and steps of eight columns each of them takes (0: any number); rows side by side in a workgroup where one wave holds a row.
struct RowShape {
    int threads, steps, beside;
};
RowShape row_shape(int cols)
{
    const int eights = (cols + 7) / 8, waves = (eights + 63) / 64;
    if (waves == 1) return {64, 1, 4};
    if (waves <= 16) return {64 * waves, 1, 1};
    if (waves <= 32) return {64 * ((waves + 1) / 2), 2, 1};
    return {1024, 0, 1};
}
template <class F> void by_steps(int steps, F f)
{
    if (steps == 1) f(std::integral_constant<int, 1>());
    else if (steps == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 0>());
}
template <class F> void by_function(int function, int gated, F f)
{
    auto with = [&](auto g) {
        if (function == XNOR_RELU) f(std::integral_constant<int, XNOR_RELU>(), g);
        else if (function == XNOR_GELU) f(std::integral_constant<int, XNOR_GELU>(), g);
        else f(std::integral_constant<int, XNOR_SILU>(), g);
    };
    if (gated) with(std::true_type());
    else with(std::false_type());
}

}  // namespace

xnor_status launch_q8_rows(const void *x, long long x_stride, int8_t *q, float *scale, int rows, int cols, int group, int type, hipStream_t stream)
{
    const RowArgs a{x, nullptr, q, nullptr, scale, nullptr, x_stride, rows, cols, group, 0};
    const RowShape s = row_shape(cols);
    const dim3 grid((unsigned)((rows + s.beside - 1) / s.beside)), block((unsigned)s.threads, (unsigned)s.beside);
    by_type(type, [&](auto t) { by_steps(s.steps, [&](auto n) { q8_rows_kernel<t(), n()><<<grid, block, 0, stream>>>(a); }); });
    return hip_status(hipGetLastError());
}

xnor_status launch_activation_q8(const void *x, long long x_stride, void *y, int8_t *q, float *scale, int8_t *kept, float *kept_scale, int rows, int cols,
                                 int group, int kept_group, int function, int gated, int type, hipStream_t stream)
{
    if (kept && gated && cols % std::max(8, kept_group)) {
        if (xnor_status e = launch_q8_rows(x, x_stride, kept, kept_scale, rows, 2 * cols, kept_group, type, stream)) return e;
        kept = nullptr;
        if (!y && !q) return XNOR_OK;
    }
    const RowArgs a{x, y, q, kept, scale, kept_scale, x_stride, rows, cols, group, kept_group};
    const RowShape s = row_shape(cols);
    const dim3 grid((unsigned)((rows + s.beside - 1) / s.beside)), block((unsigned)s.threads, (unsigned)s.beside);
    by_type(type, [&](auto t) {
        by_function(function, gated, [&](auto f, auto g) {
            by_steps(s.steps, [&](auto n) { activation_kernel<t(), f(), g(), n()><<<grid, block, 0, stream>>>(a); });
        });
    });
    return hip_status(hipGetLastError());
}

xnor_status launch_activation_backward(const int8_t *kept, const float *kept_scale, const void *g_y, long long g_stride, void *g_x, int rows, int cols,
                                       int kept_group, int function, int gated, int type, hipStream_t stream)
{
    const int eights = (cols + 7) / 8, wide = cols << gated, threads = std::min((eights + 63) / 64 * 64, 256), beside = 256 / threads;
    const int per_row = (eights + threads - 1) / threads;
    const BackwardArgs a{kept, kept_scale, g_y, g_x, g_stride, rows, cols, kept_group ? __builtin_ctz((unsigned)kept_group) : 31,
                         kept_group ? (wide + kept_group - 1) / kept_group : 1, per_row};
    const long long count = (long long)((rows + beside - 1) / beside) * per_row;
    if (count >= 0xffffff00LL / 256) return XNOR_ERR_SHAPE;
    const dim3 grid((unsigned)count), block((unsigned)threads, (unsigned)beside);
    by_type(type, [&](auto t) { by_function(function, gated, [&](auto f, auto g) { activation_grad_kernel<t(), f(), g()><<<grid, block, 0, stream>>>(a); }); });
    return hip_status(hipGetLastError());
}

}  // namespace xnor
