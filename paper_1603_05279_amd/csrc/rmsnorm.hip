// Residual addition, root-mean-square norm and 8-bit rounding of rows, and the norm's backward pass (contracts: xnor_lowbit.h).
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr float TINY = 0x1p-100f;           // groups whose largest magnitude is below hold zeros

// Sum over the threads of a row (blockDim.x, whole waves), the same value in all of them; `slots` holds a float per wave of the row.
__device__ __forceinline__ float row_sum(float v, float *slots)
{
    v = wave_sum(v);
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slots[wave] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < waves; ++i) s += slots[i];
    return s;
}

struct NormArgs {
    const void *x, *residual;
    const float *weight;
    void *sum_out;
    int8_t *q;
    float *scale;
    void *values;
    float *rstd;
    long long x_stride, residual_stride;
    int cols, group, groups;
    float eps;
};

// One row per workgroup, held in registers: thread t keeps the eight columns from 8 * (t + i * threads) on for i < STEPS.  The squares and
// the largest |t| of a whole row meet in LDS behind one barrier; a group of 32, 64 or 128 columns belongs to 4, 8 or 16 neighbouring lanes,
// which exchange its maximum.  The maximum is taken over the bit patterns of |t|, which order like the values and put infinities and NaN last.
// What bounds it: the memory (2048 x 4096 bfloat16 to sum and values 16 us, 67 MB, 4.2 TB/s with the launch; 2048 x 9216 33 us, 4.6 TB/s); a single row
// the launch and one trip to memory (1 x 4096 4.4 us).
template <int TYPE, int STEPS>
__global__ __launch_bounds__(1024) void rmsnorm_q8_kernel(NormArgs a)
{
    typedef real_t<TYPE> T;
    __shared__ float sums[16];
    __shared__ uint32_t tops[16];
    const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const size_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * (size_t)a.x_stride;
    const T *r = static_cast<const T *>(a.residual) + (a.residual ? row * (size_t)a.residual_stride : 0);
    float t[STEPS][8];
    float squares = 0.0f;
    {
        Real8<TYPE> xv[STEPS], rv[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 8 * (tid + i * (int)blockDim.x);
            xv[i].load(x + c, a.cols - c);
            if (a.residual) rv[i].load(r + c, a.cols - c);
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 8 * (tid + i * (int)blockDim.x);
            Real8<TYPE> out;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = a.residual ? xv[i][j] + rv[i][j] : xv[i][j];
                t[i][j] = h;
                out.v[j] = (T)h;
                squares += h * h;
            }
            if (a.sum_out) out.store(static_cast<T *>(a.sum_out) + row * a.cols + c, a.cols - c);
        }
    }
    uint32_t top[STEPS], row_top = 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = 8 * (tid + i * (int)blockDim.x);
        top[i] = 0;
        Real8<XNOR_F32> w;
        if (a.weight) w.load(a.weight + c, a.cols - c);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (a.weight) t[i][j] *= w[j];
            top[i] = max(top[i], __float_as_uint(t[i][j]) & 0x7fffffffu);
        }
        row_top = max(row_top, top[i]);
    }
    squares = wave_sum(squares);
    if (a.group == 0) row_top = wave_max(row_top);
    if (waves > 1) {
        if (lane == 0) {
            sums[tid >> 6] = squares;
            tops[tid >> 6] = row_top;
        }
        __syncthreads();
        squares = 0.0f;
        for (int i = 0; i < waves; ++i) {
            squares += sums[i];
            if (a.group == 0) row_top = max(row_top, tops[i]);
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(squares / (float)a.cols + a.eps);
    if (a.rstd && tid == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = 8 * (tid + i * (int)blockDim.x), n = a.cols - c;
        uint32_t bits = row_top;
        if (a.group) {
            bits = top[i];
            for (int s = a.group / 16; s > 0; s >>= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, s, 64));
        }
        const float largest = __uint_as_float(bits);
        const bool finite = bits < 0x7f800000u;
        const float factor = finite && largest >= TINY ? 127.0f / largest : 0.0f;
        float scale = (largest >= TINY ? largest : 0.0f) * rstd * (1.0f / 127.0f);
        if (!finite) scale = __builtin_nanf("");
        union {
            int8_t b[8];
            uint32_t w[2];
        } q;
        Real8<TYPE> values;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = finite ? __builtin_rintf(t[i][j] * factor) : 0.0f;
            q.b[j] = (int8_t)(int)f;
            values.v[j] = (T)(f * scale);
        }
        if (n <= 0) continue;
        if (a.scale && (a.group ? (c & (a.group - 1)) == 0 : c == 0)) a.scale[row * a.groups + (a.group ? c / a.group : 0)] = scale;
        if (a.q) {
            int8_t *p = a.q + row * a.cols + c;
            if (n >= 8) {
                typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(1)));
                *reinterpret_cast<words2 *>(p) = words2{q.w[0], q.w[1]};
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) p[j] = q.b[j];
            }
        }
        if (a.values) values.store(static_cast<T *>(a.values) + row * a.cols + c, n);
    }
}

struct NormGradArgs {
    const void *h, *g, *g_sum;
    const float *rstd, *weight;
    void *g_h;
    float *partial;                 // [gridDim.x][cols], NULL: g_weight is not asked for
    long long h_stride, g_stride, g_sum_stride;
    int rows, cols;
};

// blockDim.y rows at a time, each by blockDim.x threads (as in the forward kernel), and every gridDim.x-th such set per workgroup: a thread meets the
// same columns of each, whose shares of g_weight stay in its registers until the end, when those of the rows side by side are added in LDS.
// What bounds it: the memory, and a barrier per row (2048 x 9216 bfloat16 42 us with g_weight's sum, 151 MB, 3.6 TB/s; 2048 x 8192 float32 61 us, 4.4).
// A row read while the one before is worked on: 44 and 61 us.
template <int TYPE, int STEPS>
__global__ __launch_bounds__(1024) void rmsnorm_grad_kernel(NormGradArgs a)
{
    typedef real_t<TYPE> T;
    __shared__ float sums[2][16];
    extern __shared__ __attribute__((aligned(16))) float side[];               // [blockDim.y - 1][cols]
    const int tid = threadIdx.x, beside = __builtin_amdgcn_readfirstlane(threadIdx.y);      // (a row's threads are whole waves)
    float gw[STEPS][8];
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) gw[i][j] = 0.0f;
    int turn = 0;
    for (int first = blockIdx.x * (int)blockDim.y; first < a.rows; first += gridDim.x * blockDim.y, turn ^= 1) {
        const bool real = first + beside < a.rows;      // (threads past the last row take it once more, and leave nothing)
        const int row = real ? first + beside : a.rows - 1;
        const T *h = static_cast<const T *>(a.h) + (size_t)row * a.h_stride;
        const T *g = static_cast<const T *>(a.g) + (size_t)row * a.g_stride;
        const T *gs = static_cast<const T *>(a.g_sum) + (a.g_sum ? (size_t)row * a.g_sum_stride : 0);
        const float rstd = a.rstd[row];
        constexpr bool HELD = STEPS < 4;                // (the longest rows are read twice: their registers hold the shares of g_weight)
        Real8<TYPE> hv[STEPS], gv[STEPS], sv[STEPS];
        auto load = [&](int i) {
            const int c = 8 * (tid + i * (int)blockDim.x);
            hv[i].load(h + c, a.cols - c);
            gv[i].load(g + c, a.cols - c);
            if (a.g_sum) sv[i].load(gs + c, a.cols - c);
        };
        if (HELD)
#pragma unroll
            for (int i = 0; i < STEPS; ++i) load(i);
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 8 * (tid + i * (int)blockDim.x);
            if (!HELD) {                                // (one step's values at a time, and none kept for the second time)
                asm volatile("" : "+s"(h), "+s"(g), "+s"(gs) : : "memory");
                load(i);
            }
            Real8<XNOR_F32> w;
            if (a.weight) w.load(a.weight + c, a.cols - c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = hv[i][j] * rstd, p = gv[i][j] * n;
                if (real) gw[i][j] += p;
                dot += a.weight ? p * w[j] : p;
            }
        }
        dot = row_sum(dot, sums[turn] + beside * (blockDim.x >> 6)) / (float)a.cols;
        if (!real) continue;
        T *out = static_cast<T *>(a.g_h) + (size_t)row * a.cols;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 8 * (tid + i * (int)blockDim.x);
            if (!HELD) {                                // (one step's values at a time, and none kept for the second time)
                asm volatile("" : "+s"(h), "+s"(g), "+s"(gs) : : "memory");
                load(i);
            }
            Real8<XNOR_F32> w;
            if (a.weight) w.load(a.weight + c, a.cols - c);
            Real8<TYPE> o;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = hv[i][j] * rstd, wg = a.weight ? gv[i][j] * w[j] : gv[i][j];
                const float v = rstd * (wg - n * dot);
                o.v[j] = (T)(a.g_sum ? v + sv[i][j] : v);
            }
            o.store(out + c, a.cols - c);
        }
    }
    if (!a.partial) return;
    if (blockDim.y > 1) {
        if (beside)
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = 8 * (tid + i * (int)blockDim.x) + j;
                    if (c < a.cols) side[(beside - 1) * a.cols + c] = gw[i][j];
                }
        __syncthreads();
        if (beside) return;
        for (int k = 0; k < (int)blockDim.y - 1; ++k)
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = 8 * (tid + i * (int)blockDim.x) + j;
                    if (c < a.cols) gw[i][j] += side[k * a.cols + c];
                }
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = 8 * (tid + i * (int)blockDim.x);
        Real8<XNOR_F32> o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = gw[i][j];
        o.store(a.partial + (size_t)blockIdx.x * a.cols + c, a.cols - c);
    }
}

// g_weight = the workgroups' shares added: 64 columns per workgroup, its 16 waves take every 16th share, and the first adds theirs (in one order, whatever
// workgroup was sooner).  What bounds it: one trip to memory (256 shares of 9216 columns 4.2 us).
__global__ __launch_bounds__(1024) void rmsnorm_grad_sum_kernel(const float *__restrict__ partial, float *__restrict__ g_weight, int parts,
                                                                int cols)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 16
        for (int p = wave; p < parts; p += 16) s += partial[(size_t)p * cols + c];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= cols) return;
#pragma unroll
    for (int p = 1; p < 16; ++p) s += sums[p][lane];
    g_weight[c] = s;
}

// Steps of eight columns per thread and threads per row.
struct RowShape {
    int steps, threads;
};
RowShape row_shape(int cols)
{
    const int eights = (cols + 7) / 8, steps = eights <= 512 ? 1 : eights <= 2048 ? 2 : 4;
    return {steps, 64 * ((eights + 64 * steps - 1) / (64 * steps))};
}

template <class F> void by_steps(int steps, F f)
{
    if (steps == 1) f(std::integral_constant<int, 1>());
    else if (steps == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 4>());
}

}  // namespace

// How the backward pass shares out its rows: eight waves of rows side by side (a row's trip to memory and back would be all that a narrow row's
// workgroup waits for), and as many workgroups as take the same number of turns each, or one less: two per CU, one of the widest rows, whose shares of
// g_weight weigh more than what a second workgroup hides.  8000 x 100 float32 one row at a time 31 us, eight 12; 2048 x 9216 bfloat16 two per CU 45, one 42;
// 2048 x 4096 18 and 20.
struct GradShape {
    int beside, parts;
};
static int grad_most(int cols) { return row_shape(cols).threads > 512 ? 256 : 512; }
static GradShape grad_shape(int rows, int cols)
{
    if (rows == 0) return {1, 0};
    const int waves = row_shape(cols).threads / 64, beside = std::max(1, 8 / waves), most = grad_most(cols);
    const int sets = (rows + beside - 1) / beside, turns = (sets + most - 1) / most;
    return {beside, (sets + turns - 1) / turns};
}
// Enough for up to `rows` rows: an even share of the turns takes fewer workgroups, never more.
size_t rmsnorm_grad_workspace_bytes(int rows, int cols)
{
    const GradShape s = grad_shape(rows, cols);
    return (size_t)std::min((rows + s.beside - 1) / s.beside, grad_most(cols)) * cols * sizeof(float);
}

xnor_status launch_rmsnorm_q8(const void *x, long long x_stride, const void *residual, long long residual_stride, const float *weight,
                              void *sum_out, int8_t *q, float *scale, void *values, float *rstd, int rows, int cols, int group, int type,
                              float eps, hipStream_t stream)
{
    const NormArgs a{x, residual, weight, sum_out, q, scale, values, rstd, x_stride, residual_stride, cols, group,
                     group ? (cols + group - 1) / group : 1, eps};
    const RowShape s = row_shape(cols);
    by_type(type, [&](auto t) {
        by_steps(s.steps, [&](auto n) { rmsnorm_q8_kernel<t(), n()><<<dim3((unsigned)rows), dim3((unsigned)s.threads), 0, stream>>>(a); });
    });
    return hip_status(hipGetLastError());
}

xnor_status launch_rmsnorm_backward(const void *h, long long h_stride, const float *rstd, const float *weight, const void *g, long long g_stride,
                                    const void *g_sum, long long g_sum_stride, void *g_h, float *g_weight, void *workspace, int rows, int cols,
                                    int type, hipStream_t stream)
{
    const GradShape shape = grad_shape(rows, cols);
    const int parts = shape.parts;
    if (rows > 0) {
        const NormGradArgs a{h, g, g_sum, rstd, weight, g_h, g_weight ? static_cast<float *>(workspace) : nullptr, h_stride, g_stride,
                             g_sum_stride, rows, cols};
        const RowShape s = row_shape(cols);
        by_type(type, [&](auto t) {
            by_steps(s.steps, [&](auto n) {
                rmsnorm_grad_kernel<t(), n()><<<dim3((unsigned)parts), dim3((unsigned)s.threads, (unsigned)shape.beside),
                                                (size_t)(shape.beside - 1) * cols * sizeof(float), stream>>>(a);
            });
        });
        if (xnor_status e = hip_status(hipGetLastError())) return e;
    }
    if (!g_weight) return XNOR_OK;
    rmsnorm_grad_sum_kernel<<<dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, stream>>>(static_cast<const float *>(workspace), g_weight, parts,
                                                                                             cols);
    return hip_status(hipGetLastError());
}

}  // namespace xnor
