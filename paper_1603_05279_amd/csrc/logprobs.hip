// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their backward pass (contracts: xnor_lowbit.h).
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr int THREADS = 256, STEPS = 4, CHUNK = THREADS * 8 * STEPS;      // logits that a workgroup holds in registers at a time
constexpr int MOST_PARTS = 64, MOST_TOP = 32;
constexpr int GROUP_LANES = 4, GROUPS = THREADS / GROUP_LANES;            // threads whose largest logits are compared as one
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

// A running softmax: the largest logit m, s = sum exp(l - m) and t = sum exp(l - m) (l - m); entropy = log s - t / s.  The terms of t are
// differences, so masks of any magnitude leave it finite.
struct Stats {
    float m, s, t;
};
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }
// s and t of a, whose largest is a.m, for a largest logit m >= a.m instead
__device__ __forceinline__ Stats rescaled(Stats a, float m)
{
    const float d = a.m - m, f = exp_of(d);
    const bool some = d > -100.0f;                      // (else nothing is left of it, or nothing was summed: -inf on both sides)
    return {m, some ? f * a.s : a.s != a.s ? a.s : 0.0f, some ? f * __builtin_fmaf(d, a.s, a.t) : 0.0f};
}
// Statistics of a wave in all its lanes.
__device__ __forceinline__ Stats wave_merged(Stats a)
{
    float m = a.m;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    a = rescaled(a, m);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        a.s += __shfl_xor(a.s, d, 64);
        a.t += __shfl_xor(a.t, d, 64);
    }
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

// A wave's own writes to LDS, before its reads.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct TopLds {
    key_t list[MOST_TOP];            // the best so far, in order; filled up with none_key()
    key_t group[GROUPS];
    uint32_t short_group[GROUPS];
    int count;                  // of found
    key_t found[];              // up to top * parts
};

// The next float above v (finite; +0 above -0).
__device__ __forceinline__ float above(float v)
{
    const uint32_t u = __float_as_uint(v + 0.0f);
    return __uint_as_float(u & 0x80000000u ? u - 1 : u + 1);
}

// The upper half of a key with 6 bits less, and in their place the group's number: short keys that differ.
__device__ __forceinline__ uint32_t short_key(uint32_t upper, int group) { return (upper & ~63u) | (uint32_t)(63 - group); }

// A value that at least `top` of the 64 groups reach with their largest, from their short keys in LDS (every wave finds it by itself), as the upper
// half of a key.
__device__ __forceinline__ uint32_t short_rank(const uint32_t *groups, int top)
{
    const uint32_t g = groups[threadIdx.x & 63];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < GROUPS; i += 4) {
        const uint4 o = *reinterpret_cast<const uint4 *>(groups + i);
        rank += (o.x > g ? 1 : 0) + (o.y > g ? 1 : 0) + (o.z > g ? 1 : 0) + (o.w > g ? 1 : 0);
    }
    const int who = __builtin_ctzll(__ballot(rank == top - 1));
    return (uint32_t)__builtin_amdgcn_readlane((int)g, who) & ~63u;
}

// The top-th largest of the 64 different keys in t.group (every wave finds it by itself).
__device__ __forceinline__ key_t group_rank(const TopLds &t, int top)
{
    const int lane = threadIdx.x & 63;
    const key_t g = t.group[lane];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        const key_t o = t.group[i];
        rank += o > g ? 1 : 0;
    }
    const int who = __builtin_ctzll(__ballot(rank == top - 1));
    return (key_t)__shfl((long long)g, who, 64);
}
// The top-th largest of the groups' largest keys: at least `top` keys are not below it, and those that are not belong to `top` groups.
__device__ __forceinline__ key_t group_threshold(TopLds &t, key_t mine, int top)
{
#pragma unroll
    for (int d = 1; d < GROUP_LANES; d <<= 1) {
        const key_t o = (key_t)__shfl_xor((long long)mine, d, 64);
        mine = o > mine ? o : mine;
    }
    if (threadIdx.x % GROUP_LANES == 0) t.group[threadIdx.x / GROUP_LANES] = mine ? mine : threadIdx.x;        // (a key of its own, below all others)
    __syncthreads();
    return group_rank(t, top);
}

// list = the `top` largest of found[0 .. n), in order; called by all threads, found and n settled behind a barrier.
__device__ __forceinline__ void select_top(TopLds &t, int n, int top)
{
    // a long list is thinned out first: 32 of 64 groups can hold what is not below the threshold, so its length falls to half or less
    while (n > THREADS) {
        constexpr int MOST = MOST_PARTS * MOST_TOP / THREADS;
        key_t best = 0;
        for (int i = threadIdx.x; i < n; i += THREADS) best = max(best, t.found[i]);
        __syncthreads();                                        // (t.group is read no more)
        const key_t least = group_threshold(t, best, top);
        uint32_t keep = 0;
        for (int i = 0; i < MOST; ++i) {
            const int at = threadIdx.x + i * THREADS;
            if (at < n && t.found[at] >= least) keep |= 1u << i;
        }
        if (threadIdx.x == 0) t.count = 0;
        __syncthreads();
        // moved to places below their own or that others have left: through registers, a round of places at a time
        for (int i = 0; i * THREADS < n; ++i) {
            const bool mine = keep >> i & 1u;
            const key_t k = mine ? t.found[threadIdx.x + i * THREADS] : 0;
            __syncthreads();
            if (mine) t.found[atomicAdd(&t.count, 1)] = k;
            __syncthreads();
        }
        n = t.count;
        __syncthreads();
    }
    // ranks by counting: keys differ, so every rank is taken once
    const int i = threadIdx.x;
    const key_t mine = i < n ? t.found[i] : 0;
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += t.found[j] > mine ? 1 : 0;
    if (i < n && rank < top) t.list[rank] = mine;
    if (i >= n && i < top) t.list[i] = none_key();
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

// The logit of a thread's own given token, fetched while the row is read.
struct Given {
    bool real;
    float logit;
};
template <int TYPE> __device__ __forceinline__ Given given_at(const LogprobArgs &a, size_t row, int i)
{
    if (i >= a.given) return {false, 0.0f};
    const long long token = token_at(a.tokens, a.token_bytes, row * a.given + i);
    const bool real = token >= 0 && token < a.vocab;
    return {real, real ? (float)(static_cast<const real_t<TYPE> *>(a.logits) + row * (size_t)a.stride)[token] : 0.0f};
}

// A row's results from its statistics and the list of alternatives, by the workgroup or, WIDTH = 64, a wave of it.
template <int TYPE, int WIDTH = THREADS>
__device__ __forceinline__ void finish_row(const LogprobArgs &a, size_t row, Stats st, const key_t *list, Given own)
{
    const int i = threadIdx.x % WIDTH;
    const bool empty = st.m == -__builtin_inff() && !(st.s != st.s);
    // (the sum holds the largest logit's own term, 1: below it is a rounding, which would make its log probability positive.  Likewise the entropy.  A NaN stays)
    const float log_s = empty || st.s < 1.0f ? 0.0f : __builtin_logf(st.s), base = empty ? 0.0f : st.m;
    if (i == 0) {
        if (a.lse) a.lse[row] = empty ? -__builtin_inff() : base + log_s;
        if (a.shift) {
            a.shift[2 * row] = st.m;
            a.shift[2 * row + 1] = log_s;
        }
        const float entropy = log_s - st.t / st.s;
        if (a.entropy) a.entropy[row] = empty || entropy < 0.0f ? 0.0f : entropy;
    }
    for (int g = i; g < a.given; g += WIDTH) {
        if (g >= WIDTH) own = given_at<TYPE>(a, row, g);
        a.logprob[row * a.given + g] = own.real ? (own.logit - base) - log_s : 0.0f;
    }
    if (i < a.top) {
        const bool real = list[i] > none_key() && log_s == log_s;
        a.top_index[row * a.top + i] = real ? (int32_t)index_of(list[i]) : -1;
        a.top_logprob[row * a.top + i] = real ? (value_of(list[i]) - base) - log_s : log_s == log_s ? -__builtin_inff() : log_s;
    }
}

// `raw` (largest m) taken into a thread's statistics.
template <int TYPE, int HELD, bool ENTROPY> __device__ __forceinline__ void take(Stats &st, const Real8<TYPE> (&raw)[HELD], float m)
{
    if (m > st.m) st = rescaled(st, m);
    if (__builtin_fabsf(st.m) < 1024.0f) {
        // in powers of 2, one operation for the difference: exp(l - m) = 2^(l c - m c) with c = log2 e.  m c rounds; what it lost (below
        // 2^-13 here) is one factor of all terms, 1 - lost log 2 to 2^-27
        const float mc = st.m * LOG2E, lost = __builtin_fmaf(st.m, LOG2E, -mc);
        float s[2] = {0.0f, 0.0f}, t[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = __builtin_fmaf(raw[i][j], LOG2E, -mc), e = __builtin_amdgcn_exp2f(d);
                s[j & 1] += e;
                if (ENTROPY) t[j & 1] = __builtin_fmaf(e, fmaxf(d, -300.0f), t[j & 1]);      // (e = 0 from there on, also for -inf)
            }
        const float some = s[0] + s[1], back = 1.0f - lost * LN2;
        st.s = __builtin_fmaf(some, back, st.s);
        if (ENTROPY) st.t = __builtin_fmaf((t[0] + t[1] - lost * some) * LN2, back, st.t);
    } else {                                                // (only masks so far, or logits of an unusual size)
        const float base = st.m == -__builtin_inff() ? 0.0f : st.m;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = raw[i][j] - base, e = exp_of(d);
                st.s += e;
                if (ENTROPY) st.t = __builtin_fmaf(e, fmaxf(d, -200.0f), st.t);
            }
    }
}

// Wide rows whose alternatives nobody asks for.  A workgroup takes one part of a row (per_part logits; parts = 1: the row) chunk by chunk, the next chunk's
// loads ahead of the sums; each thread keeps statistics of its own logits.  What bounds it: the memory (4096 x 32000 bfloat16 with entropy 52 us, 5.0 TB/s; 71 right behind a
// backward pass, whose last writes are on their way),
// for few rows two launches and their trips to memory (1 x 128000 6.7 us).
template <int TYPE, bool ENTROPY>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(LogprobArgs a)
{
    typedef real_t<TYPE> T;
    __shared__ Stats wave_stats[THREADS / 64];
    const int tid = threadIdx.x;
    const size_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const int first = part * a.per_part, last = min(first + a.per_part, a.vocab);
    const T *l = static_cast<const T *>(a.logits) + row * (size_t)a.stride;
    const Given own = a.parts == 1 ? given_at<TYPE>(a, row, tid) : Given{false, 0.0f};
    Stats st{-__builtin_inff(), 0.0f, 0.0f};
    Real8<TYPE> next[STEPS];
    auto load_chunk = [&](int c0) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = c0 + 8 * (tid + i * THREADS);
            next[i].load(l + c, last - c, -__builtin_inff());
        }
    };
    load_chunk(first);
    for (int c0 = first; c0 < last; c0 += CHUNK) {
        float m = -__builtin_inff();
        Real8<TYPE> raw[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) raw[i] = next[i];
        if (c0 + CHUNK < last) load_chunk(c0 + CHUNK);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, raw[i][j]);
        take<TYPE, STEPS, ENTROPY>(st, raw, m);
    }
    st = wave_merged(st);
    if ((tid & 63) == 0) wave_stats[tid >> 6] = st;
    __syncthreads();
    {
        float m = wave_stats[0].m, s = 0.0f, t = 0.0f;
#pragma unroll
        for (int i = 1; i < THREADS / 64; ++i) m = fmaxf(m, wave_stats[i].m);
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) {
            const Stats w = rescaled(wave_stats[i], m);
            s += w.s;
            t += w.t;
        }
        st = {m, s, t};
    }
    if (a.parts == 1) finish_row<TYPE>(a, row, st, nullptr, own);
    else if (tid == 0) a.part_stats[blockIdx.x] = st;
}

// The parts of a row joined, in their order.  Each part's list is in order: the top-th of 64 of the lists' first keys bounds the alternatives from below.
// What bounds it: a launch and a chain of trips to memory and LDS (63 parts with 20 alternatives each 4.4 us).
template <int TYPE>
__global__ __launch_bounds__(THREADS) void logprobs_join_kernel(LogprobArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    TopLds &top = *reinterpret_cast<TopLds *>(smem);
    const int tid = threadIdx.x, n = a.parts * a.top;
    const size_t row = blockIdx.x;
    constexpr int MOST = MOST_PARTS * MOST_TOP / THREADS;
    Stats st{-__builtin_inff(), 0.0f, 0.0f};
    if ((tid & 63) < a.parts) st = a.part_stats[row * a.parts + (tid & 63)];      // (every wave joins them all)
    key_t first = none_key(), mine[MOST];
    if (a.top) {
        const int list = tid % a.parts, at = tid / a.parts;
        if (tid < 64 && at < min(a.top, 64 / a.parts)) first = a.part_top[row * n + (size_t)list * a.top + at];
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int at = tid + i * THREADS;
            mine[i] = at < n ? a.part_top[row * n + at] : 0;
        }
    }
    const Given own = given_at<TYPE>(a, row, tid);
    st = wave_merged(st);
    if (a.top) {
        if (tid < GROUPS) top.short_group[tid] = short_key((uint32_t)(first >> 32), tid);
        if (tid == 0) top.count = 0;
        __syncthreads();
        const key_t least = max((key_t)short_rank(top.short_group, a.top) << 32, none_key() + 1);
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (mine[i] >= least) top.found[atomicAdd(&top.count, 1)] = mine[i];
        __syncthreads();
        select_top(top, top.count, a.top);
    }
    finish_row<TYPE>(a, row, st, top.list, own);
}

// Rows whose alternatives are wanted, and narrow ones: a wave takes a part of a row (parts = 1: the row), 64 * 8 * HELD logits at a time in registers
// (LOOP: more than once, the next ones' loads ahead), without barriers.  Each lane keeps statistics and the largest of its own logits; the top-th of the
// lanes' largest bounds the alternatives from below, and only a few more logits reach it (64 log 2 = 44 of any number in random order for top = 32).  Lanes
// that hold one put their logits side by side in LDS, all lanes look through them, and what reaches the bound waits in a list, whose best are ranked by
// counting once it is full and at the end.
// What bounds it: a short row's chain of latencies (1 x 1000 bfloat16 3.5 us without alternatives, 5.7 with 20); on long ones the search's instructions beside
// the exponents' (4096 x 32000 bfloat16, 20 alternatives, 66 us, 4.0 TB/s; a workgroup per row, whose barriers every chunk waits for, 90).
template <int TYPE, int HELD, bool LOOP>
__global__ __launch_bounds__(THREADS) void logprobs_wave_kernel(LogprobArgs a, int tasks)
{
    typedef real_t<TYPE> T;
    constexpr int WAVES = THREADS / 64, LIST = 256, OWN = 8 * HELD, SPAN = 64 * OWN;
    constexpr int PITCH = OWN + 16 / (int)sizeof(T);                                    // (16 bytes more: lanes in other banks)
    __shared__ __attribute__((aligned(16))) uint32_t lane_keys[WAVES][64];
    __shared__ __attribute__((aligned(16))) key_t lists[WAVES][LIST];
    __shared__ __attribute__((aligned(16))) T held[WAVES][64][PITCH];
    __shared__ uint8_t holders[WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int task = blockIdx.x * WAVES + wave;
    if (task >= tasks) return;
    const size_t row = LOOP ? task / a.parts : task;
    const int first = LOOP ? (task - (int)row * a.parts) * a.per_part : 0, last = LOOP ? min(first + a.per_part, a.vocab) : a.vocab;
    const T *l = static_cast<const T *>(a.logits) + row * (size_t)a.stride;
    Real8<TYPE> next[HELD];
    auto load = [&](int c0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = c0 + 8 * (lane + 64 * i);
            next[i].load(l + c, last - c, -__builtin_inff());
        }
    };
    load(first);
    Given own = !LOOP || a.parts == 1 ? given_at<TYPE>(a, row, lane) : Given{false, 0.0f};
    Stats st{-__builtin_inff(), 0.0f, 0.0f};
    key_t *const list = lists[wave];
    int n = 0;                                      // candidates in the list
    float bound = -3.402823466e38f, floor_value = bound;       // what the alternatives reach (-inf is none); what a logit has to reach to be looked at
    auto below = [](unsigned long long mask) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); };
    auto raise_bound = [&]() {
        lane_keys[wave][lane] = short_key((uint32_t)(key_of(st.m, 0) >> 32), lane);
        wave_fence();
        bound = fmaxf(bound, value_of((key_t)short_rank(lane_keys[wave], a.top) << 32));
        floor_value = fmaxf(floor_value, bound);
        wave_fence();
    };
    // the list's best in order: keys differ, so every rank is taken once
    auto rank_list = [&]() {
        wave_fence();
        int kept = n > 64 ? 0 : n;
        if (n > 64) raise_bound();                  // (a long list is thinned out first)
        for (int i = 0; i < n && n > 64; i += 64) {
            const key_t k = i + lane < n ? list[i + lane] : 0;
            const bool keep = i + lane < n && value_of(k) >= bound;
            const unsigned long long mask = __ballot(keep);
            wave_fence();
            if (keep) list[kept + below(mask)] = k;
            kept += __builtin_popcountll(mask);
            wave_fence();
        }
        key_t k[LIST / 64];
        int rank[LIST / 64];
#pragma unroll
        for (int i = 0; i < LIST / 64; ++i) {
            if (64 * i >= kept) break;
            k[i] = lane + 64 * i < kept ? list[lane + 64 * i] : 0;
            rank[i] = 0;
#pragma unroll 8
            for (int j = 0; j < kept; ++j) rank[i] += list[j] > k[i] ? 1 : 0;
        }
        wave_fence();
#pragma unroll
        for (int i = 0; i < LIST / 64; ++i) {
            if (64 * i >= kept) break;
            if (lane + 64 * i < kept && rank[i] < a.top) list[rank[i]] = k[i];
        }
        n = min(kept, a.top);
        wave_fence();
    };
    for (int c0 = first; c0 < last; c0 += SPAN) {
        Real8<TYPE> raw[HELD];
#pragma unroll
        for (int i = 0; i < HELD; ++i) raw[i] = next[i];
        if (LOOP && c0 + SPAN < last) load(c0 + SPAN);
        float m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, raw[i][j]);
        take<TYPE, HELD, true>(st, raw, m);
        if (a.top == 0) continue;
        unsigned long long over = __ballot(m >= floor_value);
        if (over == 0) continue;
        const bool many = __builtin_popcountll(over) > 8;       // (fewer are looked through sooner than the bound is found anew)
        if (many) {
            raise_bound();
            over = __ballot(m >= floor_value);
        }
        if (m >= floor_value) {
            const int slot = below(over);
            holders[wave][slot] = (uint8_t)lane;
#pragma unroll
            for (int i = 0; i < HELD; ++i)
#pragma unroll
                for (int q = 0; q < Real8<TYPE>::QUADS; ++q)
                    reinterpret_cast<uint4 *>(held[wave][slot])[i * Real8<TYPE>::QUADS + q] =
                        make_uint4(raw[i].quad[q][0], raw[i].quad[q][1], raw[i].quad[q][2], raw[i].quad[q][3]);
        }
        if (many) {                                 // each lane by itself
            uint32_t taken = 0;
#pragma unroll
            for (int i = 0; i < HELD; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) taken |= raw[i][j] >= floor_value ? 1u << (8 * i + j) : 0;
            int at = __builtin_popcount(taken);
            const int mine = at;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(at, d, 64);
                at += lane >= d ? o : 0;
            }
            const int found = __builtin_amdgcn_readlane(at, 63);
            if (n + found <= LIST) {
                const T *const values = held[wave][below(over)];
                wave_fence();
                for (at += n - mine; taken; taken &= taken - 1) {
                    const int bit = __builtin_ctz(taken);
                    list[at++] = key_of((float)values[bit], (uint32_t)(c0 + 8 * (lane + 64 * (bit >> 3)) + (bit & 7)));
                }
                n += found;
                continue;
            }
        }
        // few of them, or so many that they overflow the list: one after the other
        wave_fence();
        key_t least = 0;                            // (what a key has to be above once the list was ranked)
        auto rank_now = [&]() {
            rank_list();
            if (n == a.top) least = list[a.top - 1];
        };
        if (n > LIST - 64) rank_now();
        const int entries = __builtin_popcountll(over) * OWN;
        for (int e = lane; e - lane < entries; e += 64) {
            const int slot = min(e / OWN, 63), at = e % OWN;
            const float v = e < entries ? (float)held[wave][slot][at] : -__builtin_inff();
            const key_t k = key_of(v, (uint32_t)(c0 + 8 * (holders[wave][slot] + 64 * (at >> 3)) + (at & 7)));
            const bool taken = v >= floor_value && k > least;
            const unsigned long long mask = __ballot(taken);
            if (taken) list[n + below(mask)] = k;
            n += __builtin_popcountll(mask);
            if (n > LIST - 64) rank_now();
        }
        wave_fence();
        // (of what follows, only what is above the last of `top` in the list)
        if (least) floor_value = fmaxf(floor_value, above(value_of(least)));
    }
    if (a.top) rank_list();
    st = wave_merged(st);
    if (LOOP && a.parts > 1) {
        if (lane == 0) a.part_stats[task] = st;
        if (lane < a.top) a.part_top[(size_t)task * a.top + lane] = lane < n ? list[lane] : none_key();
        return;
    }
    if (lane < a.top && lane >= n) list[lane] = none_key();
    wave_fence();
    finish_row<TYPE, 64>(a, row, st, list, own);
}

struct LogprobGradArgs {
    const void *logits, *tokens;
    const float *shift, *entropy, *g_logprob, *g_entropy;
    void *g_logits;
    long long stride;
    int vocab, given, token_bytes, parts;
};

// One pass: g = -p (G + g_entropy (log p + entropy)) with G = sum g_logprob, and the tokens' own terms added before the store.
// A row, or a part of it, belongs to the WIDTH threads of a workgroup or of a wave.  What bounds it: the memory (4096 x 32000 bfloat16 97 us, read and write
// 5.4 TB/s, 84 right behind the forward pass; 300 x 50257 float32 20 us, 5.9).  Every thread looks at every given token, so many of them cost: 4 108 us, 16 194,
// 64 566, 1024 8.4 ms.
template <int TYPE, int STEPS, int WIDTH>
__global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(LogprobGradArgs a, int rows)
{
    typedef real_t<TYPE> T;
    const int tid = threadIdx.x % WIDTH;
    const size_t row = WIDTH == THREADS ? blockIdx.x / a.parts
                                        : (size_t)blockIdx.x * (THREADS / WIDTH) + __builtin_amdgcn_readfirstlane(threadIdx.x / WIDTH);
    if (WIDTH < THREADS && row >= (size_t)rows) return;
    const int c0 = WIDTH == THREADS ? (int)(blockIdx.x % a.parts) * CHUNK : 0;
    const T *l = static_cast<const T *>(a.logits) + row * (size_t)a.stride;
    T *out = static_cast<T *>(a.g_logits) + row * (size_t)a.vocab;
    Real8<TYPE> raw[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = c0 + 8 * (tid + i * WIDTH);
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
        const int c = c0 + 8 * (tid + i * WIDTH);
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

// Parts of a row: few rows are spread over the chip, workgroups (no alternatives) or waves.  Fewer waves leave SIMDs idle, more repeat each part's search and
// are joined in a second launch: 1500 bfloat16 rows of 32000, 20 alternatives, 40 us in two parts, 47 in one; 512 rows 22 in eight, 25 in four, 30 in two.
int logprobs_spread(int top) { return top ? 4096 : 512; }
int logprobs_parts(int rows, int vocab, int top)
{
    const int longest = (vocab + 2047) / 2048;
    if (vocab <= (top ? 64 * 8 * STEPS : CHUNK)) return 1;
    return std::max(1, std::min({longest, logprobs_spread(top) / std::max(rows, 1), MOST_PARTS}));
}
int logprobs_per_part(int vocab, int parts) { return ((vocab + parts - 1) / parts + 7) / 8 * 8; }

}  // namespace

bool logprobs_needs(int rows, int vocab, int top) { return logprobs_parts(rows, vocab, top) > 1; }

size_t logprobs_workspace_bytes(int rows, int vocab, int top)
{
    // the parts of up to `rows` rows: as many as a row has at most, and no more together than are spread over the chip
    const int each = logprobs_parts(1, vocab, top);
    return each == 1 ? 0 : (size_t)std::min((long long)rows * each, (long long)logprobs_spread(top)) * (16 + 8 * (size_t)top);
}

xnor_status launch_logprobs(const void *logits, long long stride, const void *tokens, int token_bytes, float *logprob, float *lse, float *shift, float *entropy,
                            int32_t *top_index, float *top_logprob, void *workspace, int rows, int vocab, int given, int top, int type,
                            hipStream_t stream)
{
    const int parts = logprobs_parts(rows, vocab, top);
    const LogprobArgs a{logits, tokens, logprob, lse, shift, entropy, top_index, top_logprob,
                        reinterpret_cast<Stats *>(static_cast<char *>(workspace) + (size_t)rows * parts * top * 8), static_cast<key_t *>(workspace),
                        stride, vocab, given, top, token_bytes, parts, logprobs_per_part(vocab, parts)};
    const int tasks = rows * parts;
    const dim3 threads(THREADS), all((unsigned)tasks), fours((unsigned)((tasks + THREADS / 64 - 1) / (THREADS / 64)));
    by_type(type, [&](auto t) {
        if (vocab <= 512) logprobs_wave_kernel<t(), 1, false><<<fours, threads, 0, stream>>>(a, tasks);
        else if (vocab <= 64 * 8 * STEPS) logprobs_wave_kernel<t(), STEPS, false><<<fours, threads, 0, stream>>>(a, tasks);
        else if (top) logprobs_wave_kernel<t(), STEPS, true><<<fours, threads, 0, stream>>>(a, tasks);
        else if (entropy) logprobs_kernel<t(), true><<<all, threads, 0, stream>>>(a);
        else logprobs_kernel<t(), false><<<all, threads, 0, stream>>>(a);
    });
    if (xnor_status e = hip_status(hipGetLastError())) return e;
    if (parts == 1) return XNOR_OK;
    const size_t lds = top ? sizeof(TopLds) + (size_t)top * parts * sizeof(key_t) : 0;
    by_type(type, [&](auto t) { logprobs_join_kernel<t()><<<dim3((unsigned)rows), threads, lds, stream>>>(a); });
    return hip_status(hipGetLastError());
}

xnor_status launch_logprobs_backward(const void *logits, long long stride, const void *tokens, int token_bytes, const float *shift,
                                     const float *entropy, const float *g_logprob, const float *g_entropy, void *g_logits, int rows, int vocab,
                                     int given, int type, hipStream_t stream)
{
    // rows of at most 2048 logits belong to a wave each: 4096 x 1000 bfloat16 17.5 us by workgroups
    const int parts = (vocab + CHUNK - 1) / CHUNK;
    if ((long long)rows * parts > 0xffffffffLL / THREADS) return XNOR_ERR_SHAPE;       // (threads of a launch)
    const LogprobGradArgs a{logits, tokens, shift, entropy, g_logprob, g_entropy, g_logits, stride, vocab, given, token_bytes, parts};
    const unsigned fours = (unsigned)((rows + THREADS / 64 - 1) / (THREADS / 64));
    by_type(type, [&](auto t) {
        if (vocab <= 512) logprobs_grad_kernel<t(), 1, 64><<<dim3(fours), dim3(THREADS), 0, stream>>>(a, rows);
        else if (vocab <= 2048) logprobs_grad_kernel<t(), STEPS, 64><<<dim3(fours), dim3(THREADS), 0, stream>>>(a, rows);
        else logprobs_grad_kernel<t(), STEPS, THREADS><<<dim3((unsigned)(rows * parts)), dim3(THREADS), 0, stream>>>(a, rows);
    });
    return hip_status(hipGetLastError());
}

}  // namespace xnor
