// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their backward pass (contracts: xnor_lowbit.h).
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr int THREADS = 256, STEPS = 4, CHUNK = THREADS * 8 * STEPS;      // logits that a workgroup holds in registers at a time
constexpr int GROUP_LANES = 4, GROUPS = THREADS / GROUP_LANES;            // threads whose largest logits are compared as one
constexpr float LOG2E = 1.44269504088896340736f;

// A running softmax: the largest logit m, s = sum exp(l - m) and t = sum exp(l - m) (l - m); entropy = log s - t / s.  The terms of t are
// differences, so masks of any magnitude leave it finite.
struct Stats {
    float m, s, t;
};
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }
__device__ __forceinline__ void rescale(Stats &a, float m)
{
    const float d = a.m - m;
    if (d != 0.0f) {                                    // (NaN: -inf on both sides, and nothing summed yet)
        const float f = exp_of(d);
        a.t = f > 0.0f ? f * (a.t + d * a.s) : 0.0f;
        a.s = f > 0.0f ? f * a.s : a.s != a.s ? a.s : 0.0f;
    }
    a.m = m;
}
__device__ __forceinline__ Stats merged(Stats a, Stats b)
{
    const float m = fmaxf(a.m, b.m);
    rescale(a, m);
    rescale(b, m);
    return {m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ Stats wave_merged(Stats a)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) a = merged(a, {__shfl_xor(a.m, d, 64), __shfl_xor(a.s, d, 64), __shfl_xor(a.t, d, 64)});
    return a;
}

// Alternatives are ordered by one integer: the logit's bits in an order like the values', then the lowest index first.
typedef unsigned long long key_t;
__device__ __forceinline__ key_t key_of(float v, uint32_t index)
{
    const uint32_t u = __float_as_uint(v + 0.0f);       // (-0 as +0)
    return (key_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ uint32_t index_of(key_t k) { return ~(uint32_t)k; }
__device__ __forceinline__ float value_of(key_t k)
{
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ key_t none_key() { return key_of(-__builtin_inff(), 0xffffffffu) | 0xffffffffu; }       // every real choice is above

struct TopLds {
    key_t list[32];             // the best so far, in order; filled up with none_key()
    key_t group[GROUPS];
    int count;
    key_t found[];              // up to top * GROUP_LANES * (keys per thread)
};

// The top-th largest of the groups' largest keys (every wave finds it by itself): at least `top` keys are not below it, and those that are
// not belong to `top` groups.
__device__ __forceinline__ key_t group_threshold(TopLds &t, key_t mine, int top)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < GROUP_LANES; d <<= 1) {
        const key_t o = (key_t)__shfl_xor((long long)mine, d, 64);
        mine = o > mine ? o : mine;
    }
    __syncthreads();
    if (threadIdx.x % GROUP_LANES == 0) t.group[threadIdx.x / GROUP_LANES] = mine;
    __syncthreads();
    const key_t g = t.group[lane];
    int rank = 0;
#pragma unroll 16
    for (int i = 0; i < GROUPS; ++i) {
        const key_t o = t.group[i];
        rank += o > g || (o == g && i < lane) ? 1 : 0;
    }
    const int who = __builtin_ctzll(__ballot(rank == top - 1));
    return (key_t)__shfl((long long)g, who, 64);
}

// list = the `top` largest of list and found[0 .. n); called by all threads, found and n settled behind a barrier.
__device__ void select_top(TopLds &t, int n, int top)
{
    // a long list is thinned out first: 32 of 64 groups can hold what is not below the threshold, so its length falls to half or less
    while (n > THREADS) {
        key_t best = 0;
        for (int i = threadIdx.x; i < n; i += THREADS) best = max(best, t.found[i]);
        const key_t least = group_threshold(t, best, top);
        constexpr int MOST = 32 * GROUP_LANES * 32 / THREADS;
        key_t mine[MOST];
        int have = 0;
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int at = threadIdx.x + i * THREADS;
            mine[i] = at < n ? t.found[at] : 0;
            have += mine[i] >= least ? 1 : 0;
        }
        if (threadIdx.x == 0) t.count = 0;
        __syncthreads();
        int at = have ? atomicAdd(&t.count, have) : 0;
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (mine[i] >= least) t.found[at++] = mine[i];
        __syncthreads();
        n = t.count;
        __syncthreads();
    }
    // ranks by counting: keys differ, so every rank is taken once
    const int i = threadIdx.x;
    const key_t old = i < top ? t.list[i] : 0, neu = i < n ? t.found[i] : 0;
    int rank_old = i, rank_new = 0;
    for (int j = 0; j < n; ++j) {
        const key_t o = t.found[j];
        rank_old += o > old ? 1 : 0;
        rank_new += o > neu ? 1 : 0;
    }
    for (int j = 0; j < top; ++j) rank_new += t.list[j] > neu ? 1 : 0;
    __syncthreads();
    if (i < top && rank_old < top) t.list[rank_old] = old;
    if (i < n && rank_new < top) t.list[rank_new] = neu;
    __syncthreads();
}

struct LogprobArgs {
    const void *logits, *tokens;
    float *logprob, *lse, *shift, *entropy;
    int32_t *top_index;
    float *top_logprob;
    Stats *part_stats;          // [rows][parts]
    key_t *part_top;            // [rows][parts][top]
    long long stride;
    int vocab, given, top, token_bytes, parts, per_part;
};

__device__ __forceinline__ long long token_at(const void *tokens, int bytes, size_t i)
{
    return bytes == 8 ? static_cast<const long long *>(tokens)[i] : (long long)static_cast<const int32_t *>(tokens)[i];
}

// A row's results from its statistics and the list of alternatives (all threads of the workgroup).
template <int TYPE>
__device__ void finish_row(const LogprobArgs &a, size_t row, Stats st, const key_t *list)
{
    typedef real_t<TYPE> T;
    const T *l = static_cast<const T *>(a.logits) + row * (size_t)a.stride;
    const bool empty = st.m == -__builtin_inff() && !(st.s != st.s);
    const float log_s = empty ? 0.0f : __builtin_logf(st.s), base = empty ? 0.0f : st.m;
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = empty ? -__builtin_inff() : base + log_s;
        if (a.shift) {
            a.shift[2 * row] = st.m;
            a.shift[2 * row + 1] = log_s;
        }
        if (a.entropy) a.entropy[row] = empty ? 0.0f : log_s - st.t / st.s;
    }
    for (int i = threadIdx.x; i < a.given; i += blockDim.x) {
        const long long token = token_at(a.tokens, a.token_bytes, row * a.given + i);
        a.logprob[row * a.given + i] = token >= 0 && token < a.vocab ? ((float)l[token] - base) - log_s : 0.0f;
    }
    for (int i = threadIdx.x; i < a.top; i += blockDim.x) {
        const bool real = list[i] > none_key() && log_s == log_s;
        a.top_index[row * a.top + i] = real ? (int32_t)index_of(list[i]) : -1;
        a.top_logprob[row * a.top + i] = real ? (value_of(list[i]) - base) - log_s : log_s == log_s ? -__builtin_inff() : log_s;
    }
}

// A workgroup takes one part of a row (per_part logits, whole chunks; parts = 1: the row) chunk by chunk.  Each thread keeps statistics of its
// own logits; alternatives are looked for where some thread's largest logit is above the last of the list: the logits above it, or, where
// many threads have some, those not below the top-th of the groups' largest.
template <int TYPE, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(LogprobArgs a)
{
    typedef real_t<TYPE> T;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    __shared__ Stats wave_stats[THREADS / 64];
    TopLds &top = *reinterpret_cast<TopLds *>(smem);
    const int tid = threadIdx.x;
    const size_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const int first = part * a.per_part, last = min(first + a.per_part, a.vocab);
    const T *l = static_cast<const T *>(a.logits) + row * (size_t)a.stride;
    if (TOP) {
        if (tid < 32) top.list[tid] = none_key();
        __syncthreads();
    }
    Stats st{-__builtin_inff(), 0.0f, 0.0f};
    Real8<TYPE> next[STEPS];
    auto fetch = [&](int c0) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = c0 + 8 * (tid + i * THREADS);
            next[i].load(l + c, last - c, -__builtin_inff());
        }
    };
    fetch(first);
    for (int c0 = first; c0 < last; c0 += CHUNK) {
        Real8<TYPE> raw[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) raw[i] = next[i];
        if (c0 + CHUNK < last) fetch(c0 + CHUNK);
        float m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, raw[i][j]);
        if (m > st.m) rescale(st, m);
        const float base = st.m == -__builtin_inff() ? 0.0f : st.m;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = raw[i][j] - base, e = exp_of(d);
                st.s += e;
                if (ENTROPY) st.t = __builtin_fmaf(e, fmaxf(d, -200.0f), st.t);      // (e = 0 from there on, also for -inf)
            }
        if (TOP) {
            key_t least = top.list[a.top - 1];
            float least_value = value_of(least);
            const int over = __syncthreads_count(m > least_value);
            if (over == 0) continue;
            if (over > GROUP_LANES * a.top) {
                uint32_t at = 0;
#pragma unroll
                for (int i = STEPS - 1; i >= 0; --i)
#pragma unroll
                    for (int j = 7; j >= 0; --j) at = raw[i][j] == m ? (uint32_t)(8 * i * THREADS + j) : at;
                const key_t least_here = group_threshold(top, m > least_value ? key_of(m, (uint32_t)(c0 + 8 * tid) + at) : 0, a.top);
                least = max(least, least_here - 1);                        // (keys above it are wanted)
                least_value = value_of(least);
            }
            if (tid == 0) top.count = 0;
            __syncthreads();
            if (m >= least_value)
#pragma unroll
                for (int i = 0; i < STEPS; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float v = raw[i][j];
                        if (v >= least_value) {
                            const key_t k = key_of(v, (uint32_t)(c0 + 8 * (tid + i * THREADS) + j));
                            if (k > least) top.found[atomicAdd(&top.count, 1)] = k;
                        }
                    }
            __syncthreads();
            select_top(top, top.count, a.top);
        }
    }
    st = wave_merged(st);
    if ((tid & 63) == 0) wave_stats[tid >> 6] = st;
    __syncthreads();
    st = wave_stats[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) st = merged(st, wave_stats[i]);
    if (a.parts == 1) {
        finish_row<TYPE>(a, row, st, top.list);
    } else {
        if (tid == 0) a.part_stats[blockIdx.x] = st;
        if (TOP && tid < a.top) a.part_top[(size_t)blockIdx.x * a.top + tid] = top.list[tid];
    }
}

// The parts of a row joined, in their order.
template <int TYPE>
__global__ __launch_bounds__(THREADS) void logprobs_join_kernel(LogprobArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    TopLds &top = *reinterpret_cast<TopLds *>(smem);
    const int tid = threadIdx.x;
    const size_t row = blockIdx.x;
    Stats st{-__builtin_inff(), 0.0f, 0.0f};
    if ((tid & 63) < a.parts) st = a.part_stats[row * a.parts + (tid & 63)];      // (every wave joins them all)
    st = wave_merged(st);
    if (a.top) {
        if (tid < 32) top.list[tid] = none_key();
        const int n = a.parts * a.top;
        for (int i = tid; i < n; i += THREADS) {
            const key_t k = a.part_top[row * n + i];
            top.found[i] = k > none_key() ? k : (key_t)i;                          // (fillers: keys of their own, below all others)
        }
        __syncthreads();
        select_top(top, n, a.top);
    }
    finish_row<TYPE>(a, row, st, top.list);
}

struct LogprobGradArgs {
    const void *logits, *tokens;
    const float *shift, *entropy, *g_logprob, *g_entropy;
    void *g_logits;
    long long stride;
    int vocab, given, token_bytes, parts;
};

// One pass: g = -p (G + g_entropy (log p + entropy)) with G = sum g_logprob, and the tokens' own terms added before the store.
template <int TYPE>
__global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(LogprobGradArgs a)
{
    typedef real_t<TYPE> T;
    const size_t row = blockIdx.x / a.parts;
    const int c0 = (int)(blockIdx.x % a.parts) * CHUNK;
    const T *l = static_cast<const T *>(a.logits) + row * (size_t)a.stride;
    T *out = static_cast<T *>(a.g_logits) + row * (size_t)a.vocab;
    Real8<TYPE> raw[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = c0 + 8 * ((int)threadIdx.x + i * THREADS);
        raw[i].load(l + c, a.vocab - c);
    }
    const float m = a.shift[2 * row], log_s = a.shift[2 * row + 1];
    const bool empty = m == -__builtin_inff() && log_s == log_s;
    float total = 0.0f;
    const int given = a.g_logprob ? a.given : 0;
    for (int i = 0; i < given; ++i) {
        const long long token = token_at(a.tokens, a.token_bytes, row * a.given + i);
        if (token >= 0 && token < a.vocab) total += a.g_logprob[row * a.given + i];
    }
    const float slope = a.g_entropy ? a.g_entropy[row] : 0.0f;
    // (a NaN row keeps its NaN through here: the differences below are clamped)
    const float level = empty ? 0.0f : total + (a.g_entropy ? slope * a.entropy[row] : 0.0f) + (log_s - log_s);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = c0 + 8 * ((int)threadIdx.x + i * THREADS);
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float lp = fmaxf((raw[i][j] - m) - log_s, -200.0f);      // (p = 0 from there on)
            g[j] = empty ? 0.0f : -exp_of(lp) * __builtin_fmaf(slope, lp, level);
        }
        for (int k = 0; k < given; ++k) {
            const long long at = token_at(a.tokens, a.token_bytes, row * a.given + k) - c;
            if (at >= 0 && at < 8)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (at == j && raw[i][j] > -__builtin_inff()) g[j] += a.g_logprob[row * a.given + k];
        }
        Real8<TYPE> o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = (T)g[j];
        o.store(out + c, a.vocab - c);
    }
}

// Parts of a row: few rows are spread over the chip.
int logprobs_parts(int rows, int vocab)
{
    const int longest = (vocab + 2047) / 2048;
    if (vocab <= CHUNK) return 1;
    return std::max(1, std::min({longest, 512 / std::max(rows, 1), 64}));
}
int logprobs_per_part(int vocab, int parts) { return ((vocab + parts - 1) / parts + 7) / 8 * 8; }

size_t top_lds(int top, int keys) { return top ? sizeof(TopLds) + (size_t)keys * sizeof(key_t) : 0; }

}  // namespace

size_t logprobs_workspace_bytes(int rows, int vocab, int top)
{
    const int parts = logprobs_parts(rows, vocab);
    return parts == 1 ? 0 : (size_t)rows * parts * (16 + 8 * (size_t)top);
}

xnor_status launch_logprobs(const void *logits, long long stride, const void *tokens, int token_bytes, float *logprob, float *lse, float *shift, float *entropy,
                            int32_t *top_index, float *top_logprob, void *workspace, int rows, int vocab, int given, int top, int type,
                            hipStream_t stream)
{
    const int parts = logprobs_parts(rows, vocab);
    const LogprobArgs a{logits, tokens, logprob, lse, shift, entropy, top_index, top_logprob,
                        reinterpret_cast<Stats *>(static_cast<char *>(workspace) + (size_t)rows * parts * top * 8), static_cast<key_t *>(workspace),
                        stride, vocab, given, top, token_bytes, parts, logprobs_per_part(vocab, parts)};
    const dim3 grid((unsigned)(rows * parts)), threads(THREADS);
    by_type(type, [&](auto t) {
        const size_t lds = top_lds(top, top * GROUP_LANES * 8 * STEPS);
        if (top && entropy) logprobs_kernel<t(), true, true><<<grid, threads, lds, stream>>>(a);
        else if (top) logprobs_kernel<t(), true, false><<<grid, threads, lds, stream>>>(a);
        else if (entropy) logprobs_kernel<t(), false, true><<<grid, threads, 0, stream>>>(a);
        else logprobs_kernel<t(), false, false><<<grid, threads, 0, stream>>>(a);
    });
    if (xnor_status e = hip_status(hipGetLastError())) return e;
    if (parts == 1) return XNOR_OK;
    by_type(type, [&](auto t) { logprobs_join_kernel<t()><<<dim3((unsigned)rows), threads, top_lds(top, top * parts), stream>>>(a); });
    return hip_status(hipGetLastError());
}

xnor_status launch_logprobs_backward(const void *logits, long long stride, const void *tokens, int token_bytes, const float *shift,
                                     const float *entropy, const float *g_logprob, const float *g_entropy, void *g_logits, int rows, int vocab,
                                     int given, int type, hipStream_t stream)
{
    const int parts = (vocab + CHUNK - 1) / CHUNK;
    if ((long long)rows * parts > 0xffffffffLL / THREADS) return XNOR_ERR_SHAPE;       // (threads of a launch)
    const LogprobGradArgs a{logits, tokens, shift, entropy, g_logprob, g_entropy, g_logits, stride, vocab, given, token_bytes, parts};
    by_type(type, [&](auto t) { logprobs_grad_kernel<t()><<<dim3((unsigned)(rows * parts)), dim3(THREADS), 0, stream>>>(a); });
    return hip_status(hipGetLastError());
}

}  // namespace xnor
