// Tokens drawn from rows of logits by temperature, top-k, top-p and min-p (contract: xnor_lowbit.h).
//
// A row is not sorted.  Its tokens are counted in bins by their distance to the largest logit, 128 to a factor e of the weight, with the sum of their distances within the bin.
// The counts say where top_k ends, and nearly where top_p ends and the drawn token lies: the mean distance tells a bin's weight to 1 part in 10^5.  One more pass weighs
// every token that counts, adds up what lies before the bins that these three can be in, and lists what is in them; sorted, that gives all three exactly.  Where the bins
// hold too much for the list (ties, high temperatures), each end is looked for by itself: bins by their exact weights, then bins within a bin by the bits of (logit, index),
// until one holds few tokens.
//
// Weights are integers: exp(-d / T) in 64 bits, times a power of two, rounded.  Their sums are exact and depend on no order.
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr int BINS = 4096, DIGITS = 2048, LIST = 1024, PER_OCTAVE = 256;
constexpr double NO_WEIGHT = 64 * PER_OCTAVE - 1;           // in 256ths of a factor of two: from there on weights round to 0 (2^-63)
constexpr float PER_E = 128.0f;                             // bins; the last one's tokens, 32 factors e away (2^-46), have weights that round to 0 (they have 44 bits at most)

// 2^(-i / 256)
struct Powers {
    double of[PER_OCTAVE];
    constexpr Powers() : of()
    {
        for (int i = 0; i < PER_OCTAVE; ++i) {
            const double x = i * (0x1.62e42fefa39efp-1 / PER_OCTAVE);
            double sum = 0.0;
            for (int k = 24; k > 0; --k) sum = (sum + 1.0) * (-x / k);         // e^-x - 1 by its series, the smallest terms first
            of[i] = 1.0 + sum;
        }
    }
};
__device__ const Powers powers{};

struct SampleArgs {
    const void *logits;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *logprob;
    uint8_t *work;
    long long stride;
    int rows, vocab, bits, fraction, parts;     // bits of a weight of 1, and of a distance within its bin; parts of a row in workgroups of their own
};

// A row's distances and weights.
struct Weigh {
    float top, bin_factor;
    double factor;
    int bits;
    const double *table;            // 2^(-i / 256)
    // in bins, as a real number: in 32 bits, where it never falls as the logit falls (both roundings keep the order), and that is all a bin has to do
    __device__ __forceinline__ float bins(float l) const { return (top - l) * bin_factor; }
    __device__ __forceinline__ static int bin(float b) { return (int)fminf(b, BINS - 1); }
    // in 256ths of a factor of two
    __device__ __forceinline__ double distance(float l) const { return ((double)top - (double)l) * factor; }
    // times 2^bits, rounded to a whole number; t as it is, or NO_WEIGHT where it is more.  Rounding and scaling by additions: their own instructions take four times as long.
    __device__ __forceinline__ double weight(double t) const
    {
        constexpr double c = 0x1.62e42fefa39efp-9, whole = 0x1.8p52;        // ln 2 / 256
        t = fmin(t, NO_WEIGHT);
        const double n = t + whole, x = (n - whole) - t;
        const double e = __builtin_fma(x, __builtin_fma(x, __builtin_fma(x, c * c * c / 6, c * c / 2), c), 1.0);          // (the next term: 1.4e-13 at most)
        const int i = (int)(uint32_t)__builtin_bit_cast(uint64_t, n);
        const uint64_t w = __builtin_bit_cast(uint64_t, table[i & (PER_OCTAVE - 1)] * e) + ((uint64_t)(uint32_t)(bits - (i >> 8)) << 52);
        return (__builtin_bit_cast(double, w) + 0x1p52) - 0x1p52;
    }
    __device__ __forceinline__ uint64_t whole_weight(float l) const { return (uint64_t)weight(distance(l)); }
};

// Largest first, of equal ones (0 and -0 among them) the lowest index first.
__device__ __forceinline__ uint64_t key_of(float l, int index)
{
    const uint32_t u = __float_as_uint(l + 0.0f);
    return (uint64_t)~(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)index;
}

__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t u = ~(uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

// Where the ends can be.
struct Plan {
    int last, k_first, p_first, p_last, u_first, u_last;        // the last bin that counts; the bin of top_k's end, those of top_p's, of the token (none: first > last)
    uint32_t k_before, p_before, u_before;                      // tokens before them
    int how;
};
enum { SEARCH, LIST_ENDS, LIST_ALL };                           // look for each end by itself; list what is in those bins; list all that count

// What a pass over (a part of) the row adds up: weights before those bins, and of tokens with min_p.
enum { SUM_K, SUM_P, SUM_U, SUM_MIN, COUNT_MIN, SUMS };

struct Tops {
    float wave_top[16];
};
struct Shared : Tops {
    uint64_t mass[BINS + 4];        // of a bin (estimated, or exact where the ends are looked for by themselves), then of all before it
    uint32_t count[BINS + 4];
    double table[PER_OCTAVE];
    union {
        struct {
            uint64_t digit_mass[DIGITS];
            uint32_t digit_count[DIGITS];
        };
        struct {
            uint64_t list_key[LIST], list_mass[LIST];
        };
    };
    uint64_t sums[SUMS], wave_mass[16], wave_count[16];
    uint32_t listed;
    int first[6], found_bin;
    uint64_t found_before_mass, found_before_count;
    Plan plan;
};

// What the tokens up to some place in the order amount to, that one with them.
struct Place {
    uint64_t count, mass, key;
};

// Sum over the threads before this one, and over all.
__device__ __forceinline__ uint64_t scan(uint64_t v, uint64_t *slots, uint64_t &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    uint64_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up((unsigned long long)s, d, 64);
        if (lane >= d) s += o;
    }
    if (lane == 63) slots[wave] = s;
    __syncthreads();
    uint64_t before = 0;
    all = 0;
    for (int i = 0; i < waves; ++i) {
        if (i < wave) before += slots[i];
        all += slots[i];
    }
    __syncthreads();
    return before + s - v;
}

// A row's tokens first .. last - 1.
template <int TYPE> struct Slice {
    typedef real_t<TYPE> T;
    const T *l;
    int first, last;
    // f(eight of them, the first one's index), -inf behind the end; the next eight are on their way meanwhile, and those behind them
    template <class F> __device__ __forceinline__ void eights(F f) const
    {
        const int step = 8 * blockDim.x;
        auto load = [&](int c) {
            Real8<TYPE> v;
            if (c < last) v.load(l + c, last - c, -__builtin_inff());
            return v;
        };
        int c = first + 8 * (int)threadIdx.x;
        Real8<TYPE> now = load(c), next = load(c + step);
        for (; c < last; c += step) {
            const Real8<TYPE> v = now;
            now = next;
            next = load(c + 2 * step);
            f(v, c);
        }
    }
    // f(logit, index) for every one above -inf
    template <class F> __device__ __forceinline__ void each(F f) const
    {
        eights([&](const Real8<TYPE> &v, int c) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v[j] > -__builtin_inff()) f(v[j], c + j);
        });
    }
};

// floor(f * whole) (up: the least integer not below it) for 0 <= f < 1, exactly
__device__ __forceinline__ uint64_t share(float f, uint64_t whole, bool up)
{
    const int e = __builtin_amdgcn_frexp_expf(f), shift = 24 - e;           // f = digits / 2^shift
    const uint64_t digits = (uint64_t)__builtin_amdgcn_ldexpf(f, shift);
    const unsigned __int128 product = (unsigned __int128)digits * whole;
    if (shift >= 96) return up && product != 0;
    const uint64_t down = (uint64_t)(product >> shift);
    return down + (up && ((unsigned __int128)down << shift) != product);
}

// What a row is drawn with.
struct Settings {
    float T, top_p, min_p, u;
    int top_k;
    bool bad;
    __device__ __forceinline__ Settings(const SampleArgs &a, size_t r)
    {
        T = a.temperature ? a.temperature[r] : 1.0f;
        top_p = a.top_p ? a.top_p[r] : 1.0f;
        min_p = a.min_p ? a.min_p[r] : 0.0f;
        u = a.uniform[r];
        top_k = a.top_k ? a.top_k[r] : 0;
        bad = !(T >= 0.0f) || top_p != top_p || min_p != min_p || u != u;
        u = u < 0.0f ? 0.0f : u < 1.0f ? u : 0x1.fffffep-1f;
    }
    __device__ __forceinline__ bool first_only() const { return T == 0.0f || top_k == 1; }
    __device__ __forceinline__ uint64_t top_target(uint64_t mass) const { return top_p > 0.0f ? max((unsigned long long)share(top_p, mass, true), 1ull) : 1; }
    __device__ __forceinline__ uint64_t draw_target(uint64_t mass) const { return share(u, mass, false) + 1; }
};

// The largest of some tokens, the same in all threads; a NaN where one is NaN or +inf.
template <int TYPE> __device__ __forceinline__ float top_of(Tops &s, const Slice<TYPE> &slice)
{
    constexpr int AT_ONCE = 4;
    float top = -__builtin_inff();
    bool bad = false;
    for (int c = slice.first + 8 * (int)threadIdx.x; c < slice.last; c += 8 * AT_ONCE * blockDim.x) {
        Real8<TYPE> v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int at = c + 8 * i * (int)blockDim.x;
            v[i].load(slice.l + min(at, slice.last - 1), slice.last - at, -__builtin_inff());
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top = fmaxf(top, v[i][j]);
                bad |= !(v[i][j] < __builtin_inff());
            }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const bool any_bad = __any(bad);
    if ((threadIdx.x & 63) == 0) s.wave_top[threadIdx.x >> 6] = any_bad ? __builtin_nanf("") : top;
    __syncthreads();
    top = -__builtin_inff();
    bad = false;
    for (int i = 0; i < (int)blockDim.x >> 6; ++i) {
        bad |= s.wave_top[i] != s.wave_top[i];
        top = fmaxf(top, s.wave_top[i]);
    }
    return bad ? __builtin_nanf("") : top;
}

// A row from which nothing, or only the first token can be drawn; false: another.
template <int TYPE> __device__ __forceinline__ bool simple_row(const SampleArgs &a, Shared &s, const Slice<TYPE> &row, const Settings &set, float top, size_t r)
{
    const bool bad = set.bad || top != top;
    if (bad || top == -__builtin_inff()) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = bad ? __builtin_nanf("") : -__builtin_inff();
            if (a.kept) a.kept[r] = 0;
        }
        return true;
    }
    if (!set.first_only()) return false;
    if (threadIdx.x == 0) s.listed = ~0u;
    __syncthreads();
    row.each([&](float l, int index) {
        if (l == top) atomicMin(&s.listed, (uint32_t)index);
    });
    __syncthreads();
    if (threadIdx.x == 0) {
        a.token[r] = (int)s.listed;
        if (a.logprob) a.logprob[r] = 0.0f;
        if (a.kept) a.kept[r] = 1;
    }
    return true;
}

__device__ __forceinline__ void write_drawn(const SampleArgs &a, const Weigh &w, float T, size_t r, uint64_t key, uint64_t count, uint64_t mass)
{
    a.token[r] = (int)(uint32_t)key;
    if (a.kept) a.kept[r] = (int)count;
    // (l - top) / T - log(sum): the token's weight as it is, not as it was rounded
    if (a.logprob) a.logprob[r] = fminf((float)(((double)logit_of(key) - (double)w.top) / (double)T - log(__builtin_ldexp((double)mass, -a.bits))), 0.0f);
}

__device__ __forceinline__ void make_table(Shared &s)
{
    for (int i = threadIdx.x; i < PER_OCTAVE; i += blockDim.x) s.table[i] = powers.of[i];
}

// Into s.mass: the count in the upper bits, the sum of the distances within the bin below (the highest 34 bits hold more than there are tokens).
template <int TYPE> __device__ __forceinline__ void count_bins(Shared &s, const Slice<TYPE> &slice, const Weigh &w, int fraction)
{
    for (int i = threadIdx.x; i < BINS; i += blockDim.x) s.mass[i] = 0;
    __syncthreads();
    const float steps = (float)(1 << fraction);
    slice.each([&](float l, int) {
        const float b = w.bins(l);
        const int bin = Weigh::bin(b);
        const uint32_t within = bin < BINS - 1 ? (uint32_t)((b - (float)bin) * steps) : 0;
        atomicAdd((unsigned long long *)&s.mass[bin], (1ull << 34) + within);
    });
    __syncthreads();
}
// What a bin's counts and distances stand for: weights in 2^-32, at the mean distance of its tokens (their mean weight is above that by 1 / (8 * 128^2) at most).
__device__ __forceinline__ uint64_t estimate(uint64_t counted, int bin, int fraction)
{
    const uint32_t n = (uint32_t)(counted >> 34);
    const float within = n ? ((float)(counted & 0x3ffffffffull) / (float)n + 0.5f) / (float)(1 << fraction) : 0.0f;
    return n ? (uint64_t)fmax((double)n * (double)exp2f((bin + within) * (-1.44269504f / PER_E)) * 0x1p32, 1.0) : 0;         // (a bin that holds any ends somewhere)
}

// The bins' counts and masses become those of all before.  COUNTED: s.mass holds what count_bins left.
template <bool COUNTED> __device__ __forceinline__ void add_up(Shared &s, int fraction)
{
    constexpr int PER = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    uint64_t base_c = 0, base_m = 0;
    for (int first = 0; first < BINS; first += PER * blockDim.x) {          // (once, with 1024 threads)
        const int at = first + PER * threadIdx.x;
        uint32_t c[PER], own_c = 0;
        uint64_t m[PER], own_m = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            m[i] = s.mass[at + i];
            c[i] = COUNTED ? (uint32_t)(m[i] >> 34) : s.count[at + i];
            if (COUNTED) m[i] = estimate(m[i], at + i, fraction);
            own_c += c[i];
            own_m += m[i];
        }
        uint32_t sum_c = own_c;
        uint64_t sum_m = own_m;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t oc = __shfl_up(sum_c, d, 64);
            const uint64_t om = __shfl_up((unsigned long long)sum_m, d, 64);
            if (lane >= d) {
                sum_c += oc;
                sum_m += om;
            }
        }
        if (lane == 63) {
            s.wave_count[wave] = sum_c;
            s.wave_mass[wave] = sum_m;
        }
        __syncthreads();
        uint64_t before_c = base_c + sum_c - own_c, before_m = base_m + sum_m - own_m;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i >= waves) break;
            const uint64_t wc = s.wave_count[i], wm = s.wave_mass[i];
            if (i < wave) {
                before_c += wc;
                before_m += wm;
            }
            base_c += wc;
            base_m += wm;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s.count[at + i] = (uint32_t)before_c;
            s.mass[at + i] = before_m;
            before_c += c[i];
            before_m += m[i];
        }
        if (first + PER * (int)blockDim.x >= BINS && threadIdx.x == 0) {
            s.count[BINS] = (uint32_t)base_c;
            s.mass[BINS] = base_m;
        }
        __syncthreads();
    }
}

// The bin that holds the first place where the measure reaches the target (1 .. all of it).
template <class T> __device__ __forceinline__ int bin_of(const T *before, uint64_t target)
{
    int lo = 0;
#pragma unroll
    for (int step = BINS / 2; step > 0; step >>= 1) lo = before[lo + step] < target ? lo + step : lo;
    return lo;
}

// In 256ths of a factor of two, the distance of weight min_p.
__device__ __forceinline__ double furthest_of(const Settings &set)
{
    return set.min_p > 0.0f ? fmax(-PER_OCTAVE * log2((double)set.min_p), 0.0) : __builtin_inf();
}

__device__ __forceinline__ int list_size() { return min(LIST, (int)blockDim.x); }        // (sorted by a thread each)

// From the counts and the estimated masses.  An estimate is within 1.2e-5 of the true mass (the mean distance 8e-6, float32 the rest) and half a step of the distances, so that
// a share of the whole lies within twice that of where the estimates put it.  The even lanes look below, the odd ones above.
__device__ __forceinline__ void make_plan(Shared &s, const Settings &set, int fraction)
{
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        const double width = 2.4 * (1.2e-5 + 0.5 / PER_E / (1 << fraction)), away = lane & 1 ? 1 + width : 1 - width;
        Plan p;
        p.p_first = BINS;                   // (none)
        p.p_last = p.k_first = -1;
        p.last = BINS - 1;
        p.k_before = p.p_before = 0;
        uint64_t least = s.mass[BINS], most = least;
        uint32_t wanted = 0;
        auto look = [&](double share, int &first, int &last, uint32_t &before) {
            const int bin = min(bin_of(s.mass, (uint64_t)fmin(fmax(share * (double)(lane & 1 ? most : least) * away, 1.0), (double)most)), p.last);
            first = __shfl(bin, 0, 64);
            last = __shfl(bin, 1, 64);
            before = s.count[first];
            wanted += s.count[last + 1] - before;
        };
        if (set.top_k > 0 && (uint32_t)set.top_k < s.count[BINS]) {
            p.last = p.k_first = bin_of(s.count, (uint64_t)set.top_k);
            p.k_before = s.count[p.last];
            wanted += s.count[p.last + 1] - p.k_before;
            least = s.mass[p.last];
            most = s.mass[p.last + 1];
        }
        if (set.top_p < 1.0f) {
            look(set.top_p, p.p_first, p.p_last, p.p_before);
            least = (uint64_t)fmax((double)set.top_p * (double)least * (1 - width), 0.0);
            most = min((unsigned long long)most, (unsigned long long)s.mass[p.p_last + 1]);
        }
        if (set.min_p > 0.0f) {
            const int b = (int)fmin(furthest_of(set) * (0.6931472 / PER_OCTAVE * PER_E), (double)(BINS - 1));
            least = min((unsigned long long)least, (unsigned long long)s.mass[max(b - 1, 0)]);
            most = min((unsigned long long)most, (unsigned long long)s.mass[min(b + 2, BINS)]);
        }
        look(set.u, p.u_first, p.u_last, p.u_before);
        const uint32_t fits = (uint32_t)list_size();
        p.how = s.count[p.last + 1] <= fits ? LIST_ALL : wanted <= fits ? LIST_ENDS : SEARCH;
        if (lane == 0) s.plan = p;
    }
    __syncthreads();
}

__device__ __forceinline__ void start_list(Shared &s)
{
    if (threadIdx.x < SUMS) s.sums[threadIdx.x] = 0;
    if (threadIdx.x < 6) s.first[threadIdx.x] = LIST;
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
}
// Its key; true: there was room.
__device__ __forceinline__ bool put(Shared &s, float l, int index, uint32_t &at)
{
    at = atomicAdd(&s.listed, 1u);
    if (at >= (uint32_t)list_size()) return false;
    s.list_key[at] = key_of(l, index);
    return true;
}

// Lists a slice's tokens up to the plan's last bin.
template <int TYPE> __device__ __forceinline__ void list_all(Shared &s, const Slice<TYPE> &slice, const Weigh &w)
{
    start_list(s);
    const int last = s.plan.last;
    slice.each([&](float l, int index) {
        uint32_t at;
        if (Weigh::bin(w.bins(l)) <= last) put(s, l, index, at);
    });
    __syncthreads();
}

// Weighs a slice: the sums, and the list of what lies in the plan's bins.  A thread's sums are whole numbers below 2^52 (2^44 for each of 2^8 tokens, or 2^(62 - b)
// for each of 2^(b - 10)), which a double holds.
// What bounds it: vector instructions, about 40 for a token.
template <int TYPE> __device__ __forceinline__ void weigh(Shared &s, const Slice<TYPE> &slice, const Weigh &w, const Settings &set)
{
    const Plan p = s.plan;
    start_list(s);
    const double furthest = furthest_of(set);
    // far tokens are weighed only where min_p is smaller than their weights
    const float far = set.min_p > 0.0f && furthest > 40 * PER_OCTAVE ? __builtin_inff() : BINS - 1;
    const bool by_mass = p.p_first <= p.p_last, by_weight = set.min_p > 0.0f;
    const int k_limit = p.k_first >= 0 ? p.k_first : BINS;
    const uint32_t u_wide = p.u_last - p.u_first, p_wide = by_mass ? p.p_last - p.p_first : 0;
    double sum_k = 0, sum_p = 0, sum_u = 0, sum_min = 0;
    uint32_t count_min = 0;
    slice.eights([&](const Real8<TYPE> &eight, int c) {
        Real8<TYPE> v = eight;
#pragma unroll 1
        for (int pair = 0; pair < 4; ++pair) {              // (two at a time: more of them side by side leave no registers)
bool listed[2];
            double m[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float l = v[j], b = w.bins(l);
                const int bin = Weigh::bin(b);
                const bool is = (l > -__builtin_inff()) & !(b >= far) & (bin <= p.last);
                const double t = w.distance(l);
                m[j] = w.weight(t);
                m[j] = is ? m[j] : 0.0;
                sum_k = __builtin_fma(m[j], bin < k_limit ? 1.0 : 0.0, sum_k);
                if (by_mass) sum_p = __builtin_fma(m[j], bin < p.p_first ? 1.0 : 0.0, sum_p);
                sum_u = __builtin_fma(m[j], bin < p.u_first ? 1.0 : 0.0, sum_u);
                if (by_weight) {
                    sum_min = __builtin_fma(m[j], t <= furthest ? 1.0 : 0.0, sum_min);
                    count_min += is & (t <= furthest);
                }
                listed[j] = is & (((uint32_t)(bin - p.u_first) <= u_wide) | ((uint32_t)(bin - p.p_first) <= p_wide) | (bin == p.k_first));
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (listed[j]) {
                    uint32_t at;
                    if (put(s, v[j], c + 2 * pair + j, at)) s.list_mass[at] = (uint64_t)m[j];
                }
#pragma unroll
            for (int j = 0; j < 6; ++j) v.v[j] = v.v[j + 2];
        }
    });
    auto add = [&](int i, uint64_t v) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) v += __shfl_xor((unsigned long long)v, d, 64);
        if ((threadIdx.x & 63) == 0) atomicAdd((unsigned long long *)&s.sums[i], (unsigned long long)v);
    };
    add(SUM_K, (uint64_t)sum_k);
    if (by_mass) add(SUM_P, (uint64_t)sum_p);
    add(SUM_U, (uint64_t)sum_u);
    if (by_weight) {
        add(SUM_MIN, (uint64_t)sum_min);
        add(COUNT_MIN, count_min);
    }
    __syncthreads();
}

// The listed tokens in order, one per thread: its key and weight, and the weights of the listed ones up to it, which s.list_mass holds too.
struct Listed {
    uint64_t key, own, upto;
    int n;
    template <bool WEIGHED> __device__ __forceinline__ void sort_long(Shared &s)
    {
        const int i = threadIdx.x;
        int size = 64;
        while (size < n) size *= 2;
        // a bitonic sort: partners within a wave by exchange of lanes, others through LDS
        for (int k = 2; k <= size; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                uint64_t other, others = 0;
                if (j < 64) {
                    if (i >= size) continue;                    // (whole waves)
                    other = __shfl_xor((unsigned long long)key, j, 64);
                    if (WEIGHED) others = __shfl_xor((unsigned long long)own, j, 64);
                } else {
                    __syncthreads();
                    s.list_key[i] = key;
                    if (WEIGHED) s.list_mass[i] = own;
                    __syncthreads();
                    other = s.list_key[i ^ j];
                    if (WEIGHED) others = s.list_mass[i ^ j];
                }
                const bool low = ((i & k) == 0) == ((i & j) == 0);
                if (low ? other < key : other > key) {
                    key = other;
                    own = others;
                }
            }
    }
    template <bool WEIGHED> __device__ __forceinline__ void sort(Shared &s, const Weigh &w)
    {
        const int i = threadIdx.x;
        n = min((int)s.listed, list_size());
        key = i < n ? s.list_key[i] : ~0ull;
        own = WEIGHED && i < n ? s.list_mass[i] : 0;
        if (n <= (int)blockDim.x / 2) {
            // each token's place by counting those before it, several threads to a token (256 of 1024: 2 us, 512: 7; the sort takes 15)
            int share = 2;
            while (share < 64 && 2 * share * n <= (int)blockDim.x) share *= 2;
            const int of = i / share;
            const uint64_t mine = of < n ? s.list_key[of] : 0, its = WEIGHED && of < n ? s.list_mass[of] : 0;
            int before = 0;
            for (int j = i & (share - 1); j < n; j += share) before += s.list_key[j] < mine;
            for (int d = share / 2; d > 0; d >>= 1) before += __shfl_xor(before, d, 64);
            __syncthreads();
            if (of < n && (i & (share - 1)) == 0) {
                s.list_key[before] = mine;
                if (WEIGHED) s.list_mass[before] = its;
            }
            __syncthreads();
            key = i < n ? s.list_key[i] : ~0ull;
            own = WEIGHED && i < n ? s.list_mass[i] : 0;
        } else {
            sort_long<WEIGHED>(s);
        }
        if (!WEIGHED && i < n) own = w.whole_weight(logit_of(key));
        uint64_t all;
        upto = scan(own, s.wave_mass, all) + own;
        s.list_mass[i] = upto;
        __syncthreads();
    }
    // The first thread that says yes, LIST if none; `slot` of s.first holds LIST before.
    __device__ __forceinline__ int first(Shared &s, bool yes, int slot) const
    {
        const uint64_t all = __ballot(yes);
        if (all && (threadIdx.x & 63) == 0) atomicMin(&s.first[slot], (int)threadIdx.x + __builtin_ctzll(all));
        __syncthreads();
        return s.first[slot];
    }
};

// From a list of all tokens that count.  False: it did not fit.
__device__ __forceinline__ bool draw_all(const SampleArgs &a, Shared &s, const Weigh &w, const Settings &set, uint32_t seen, size_t r)
{
    if (s.listed > (uint32_t)list_size()) return false;
    Listed l;
    l.sort<false>(s, w);
    const int i = threadIdx.x;
    int count = set.top_k > 0 && (uint32_t)set.top_k < seen ? set.top_k : (int)seen;
    uint64_t mass = s.list_mass[count - 1];
    if (set.top_p < 1.0f) count = l.first(s, i < count && l.upto >= set.top_target(mass), 0) + 1;
    if (set.min_p > 0.0f) count = min(count, l.first(s, i >= l.n || w.distance(logit_of(l.key)) > furthest_of(set), 1));
    mass = s.list_mass[count - 1];
    const int at = l.first(s, l.upto >= set.draw_target(mass), 2);
    if (i == at) write_drawn(a, w, set.T, r, l.key, count, mass);
    return true;
}

// From the sums and the list.  False: the plan did not hold what was looked for.
__device__ __forceinline__ bool draw_ends(const SampleArgs &a, Shared &s, const Weigh &w, const Settings &set, uint32_t seen, size_t r)
{
    if (s.listed > (uint32_t)list_size()) return false;
    const Plan plan = s.plan;
    Listed l;
    l.sort<true>(s, w);
    const int i = threadIdx.x, bin = i < l.n ? Weigh::bin(w.bins(logit_of(l.key))) : BINS;
    const bool by_count = plan.k_first >= 0, by_mass = plan.p_first <= plan.p_last;
    uint64_t count = seen, mass = s.sums[SUM_K];
    // what the listed ones before a bin's first weigh
    auto before = [&](int first) { return first > 0 ? s.list_mass[first - 1] : 0; };
    if (by_count) {
        const int start = l.first(s, bin >= plan.k_first, 0), at = start + (int)(set.top_k - plan.k_before) - 1;
        if (at >= l.n) return false;
        count = set.top_k;
        mass += s.list_mass[at] - before(start);
    }
    if (by_mass) {
        const int start = l.first(s, bin >= plan.p_first, 1);
        const uint64_t base = s.sums[SUM_P] - before(start), target = set.top_target(mass);
        const int at = l.first(s, bin >= plan.p_first && bin <= plan.p_last && base + l.upto >= target, 2);
        if (at >= l.n || s.sums[SUM_P] >= target) return false;
        count = plan.p_before + (at - start) + 1;
        mass = base + s.list_mass[at];
    }
    if (set.min_p > 0.0f) {
        count = min((unsigned long long)count, (unsigned long long)s.sums[COUNT_MIN]);
        mass = min((unsigned long long)mass, (unsigned long long)s.sums[SUM_MIN]);
    }
    const int start = l.first(s, bin >= plan.u_first, 3);
    const uint64_t base = s.sums[SUM_U] - before(start), target = set.draw_target(mass);
    const int at = l.first(s, bin >= plan.u_first && bin <= plan.u_last && base + l.upto >= target, 4);
    if (at >= l.n || s.sums[SUM_U] >= target) return false;
    if (i == at) write_drawn(a, w, set.T, r, l.key, count, mass);
    return true;
}

// The first place in the order where the measure reaches the target, by itself: digit by digit of (logit, index) within its bin.
template <int TYPE, bool BY_MASS> __device__ __forceinline__ Place search(Shared &s, const Slice<TYPE> &row, const Weigh &w, uint64_t target)
{
    const int bin0 = BY_MASS ? bin_of(s.mass, target) : bin_of(s.count, target);
    uint64_t before_count = s.count[bin0], before_mass = s.mass[bin0], prefix = 0, mask = 0;
    uint32_t in_bin = s.count[bin0 + 1] - s.count[bin0];
    int shift = 64;
    while (in_bin > (uint32_t)list_size()) {         // (ends: the keys differ, and the last digit is 9 bits)
        const int next = shift > 11 ? shift - 11 : 0, width = shift - next;
        __syncthreads();
        for (int i = threadIdx.x; i < DIGITS; i += blockDim.x) {
            s.digit_count[i] = 0;
            s.digit_mass[i] = 0;
        }
        __syncthreads();
        row.each([&](float l, int index) {
            const uint64_t key = key_of(l, index);
            if (Weigh::bin(w.bins(l)) != bin0 || (key & mask) != prefix) return;
            const int d = (int)(key >> next) & ((1 << width) - 1);
            atomicAdd(&s.digit_count[d], 1u);
            atomicAdd((unsigned long long *)&s.digit_mass[d], (unsigned long long)w.whole_weight(l));
        });
        __syncthreads();
        const int per = DIGITS / blockDim.x, first = threadIdx.x * per;
        uint64_t c = 0, m = 0, all;
        for (int i = 0; i < per; ++i) {
            c += s.digit_count[first + i];
            m += s.digit_mass[first + i];
        }
        uint64_t bc = before_count + scan(c, s.wave_count, all), bm = before_mass + scan(m, s.wave_mass, all);
        const uint64_t start = BY_MASS ? bm : bc;
        if (start < target && target <= start + (BY_MASS ? m : c))
            for (int i = 0; i < per; ++i) {
                const uint64_t nc = bc + s.digit_count[first + i], nm = bm + s.digit_mass[first + i];
                if ((BY_MASS ? nm : nc) >= target) {
                    s.found_bin = first + i;
                    s.found_before_count = bc;
                    s.found_before_mass = bm;
                    break;
                }
                bc = nc;
                bm = nm;
            }
        __syncthreads();
        before_count = s.found_before_count;
        before_mass = s.found_before_mass;
        prefix |= (uint64_t)s.found_bin << next;
        mask |= (uint64_t)((1u << width) - 1) << next;
        in_bin = s.digit_count[s.found_bin];
        shift = next;
    }
    __syncthreads();
    if (threadIdx.x < 6) s.first[threadIdx.x] = LIST;
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    row.each([&](float l, int index) {
        const uint64_t key = key_of(l, index);
        uint32_t at;
        if (Weigh::bin(w.bins(l)) == bin0 && (key & mask) == prefix) put(s, l, index, at);          // (in_bin of them: they fit)
    });
    __syncthreads();
    Listed l;
    l.sort<false>(s, w);
    const uint64_t rest = target - (BY_MASS ? before_mass : before_count);
    const int at = l.first(s, (BY_MASS ? l.upto : (uint64_t)threadIdx.x + 1) >= rest, 0);
    if ((int)threadIdx.x == at) s.list_key[0] = l.key;
    __syncthreads();
    const Place p{before_count + at + 1, before_mass + s.list_mass[at], s.list_key[0]};
    __syncthreads();
    return p;
}

// Every end by itself, on exact weights of all bins.
template <int TYPE> __device__ __forceinline__ void draw_searched(const SampleArgs &a, Shared &s, const Slice<TYPE> &row, const Weigh &w, const Settings &set, size_t r)
{
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += blockDim.x) {
        s.count[i] = 0;
        s.mass[i] = 0;
    }
    if (threadIdx.x < SUMS) s.sums[threadIdx.x] = 0;
    __syncthreads();
    const double furthest = furthest_of(set);
    uint64_t sum_min = 0;
    uint32_t count_min = 0;
    row.each([&](float l, int) {
        const int bin = Weigh::bin(w.bins(l));
        const uint64_t m = w.whole_weight(l);
        atomicAdd(&s.count[bin], 1u);
        atomicAdd((unsigned long long *)&s.mass[bin], (unsigned long long)m);
        if (w.distance(l) <= furthest) {
            sum_min += m;
            ++count_min;
        }
    });
    atomicAdd((unsigned long long *)&s.sums[SUM_MIN], (unsigned long long)sum_min);
    atomicAdd((unsigned long long *)&s.sums[COUNT_MIN], (unsigned long long)count_min);
    __syncthreads();
    add_up<false>(s, 0);
    uint64_t count = s.count[BINS], mass = s.mass[BINS];
    if (set.top_k > 0 && (uint64_t)set.top_k < count) {
        const Place p = search<TYPE, false>(s, row, w, (uint64_t)set.top_k);
        count = p.count;
        mass = p.mass;
    }
    if (set.top_p < 1.0f) {
        const Place p = search<TYPE, true>(s, row, w, set.top_target(mass));
        count = p.count;
        mass = p.mass;
    }
    if (set.min_p > 0.0f) {
        count = min((unsigned long long)count, (unsigned long long)s.sums[COUNT_MIN]);
        mass = min((unsigned long long)mass, (unsigned long long)s.sums[SUM_MIN]);
    }
    const Place p = search<TYPE, true>(s, row, w, set.draw_target(mass));
    if (threadIdx.x == 0) write_drawn(a, w, set.T, r, p.key, count, mass);
}

__device__ __forceinline__ Weigh weigher(const SampleArgs &a, const Shared &s, const Settings &set, float top)
{
    return Weigh{top, PER_E / set.T, PER_OCTAVE * 0x1.71547652b82fep+0 / (double)set.T, a.bits, s.table};          // log2 e
}

// From what a pass over the whole row left.
template <int TYPE> __device__ __forceinline__ void draw(const SampleArgs &a, Shared &s, const Slice<TYPE> &row, const Weigh &w, const Settings &set, uint32_t seen, size_t r)
{
    if (s.plan.how == LIST_ALL && draw_all(a, s, w, set, seen, r)) return;
    if (s.plan.how == LIST_ENDS && draw_ends(a, s, w, set, seen, r)) return;
    draw_searched(a, s, row, w, set, r);
}

// A row per workgroup.
// What bounds it: vector instructions of the row's CU: 256 x 32000 bfloat16 37 us, of which 16 weigh all tokens; 23 with a top_k of 64.
template <int TYPE> __global__ __launch_bounds__(1024) void sample_kernel(SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Shared &s = *reinterpret_cast<Shared *>(lds);
    const size_t r = blockIdx.x;
    const Slice<TYPE> row{static_cast<const real_t<TYPE> *>(a.logits) + r * (size_t)a.stride, 0, a.vocab};
    const Settings set(a, r);
    make_table(s);
    const float top = top_of(s, row);
    if (simple_row(a, s, row, set, top, r)) return;
    const Weigh w = weigher(a, s, set, top);
    if (a.vocab <= list_size() / 2) {           // (all of them at once)
        if (threadIdx.x == 0) s.plan.last = BINS - 1;
        list_all(s, row, w);
        draw_all(a, s, w, set, s.listed, r);
        return;
    }
    count_bins(s, row, w, a.fraction);
    add_up<true>(s, a.fraction);
    make_plan(s, set, a.fraction);
    const uint32_t seen = s.count[BINS];
    if (s.plan.how == LIST_ALL) list_all(s, row, w);
    else if (s.plan.how == LIST_ENDS) weigh(s, row, w, set);
    draw(a, s, row, w, set, seen, r);
}

// Few rows: a row in parts of at most 2^13 - 8 tokens, each in a workgroup of its own, and a launch for each step.  What a part leaves for the next:
struct Part {
    uint32_t bins[BINS];            // count in the upper 13 bits, the sum of 6-bit distances within the bin below
    uint64_t list_key[LIST], list_mass[LIST], sums[SUMS];
    float top;
    uint32_t listed, seen;          // seen, plan: of the first part only, for the row
    Plan plan;
};
constexpr int PART_FRACTION = 6, PART_SHIFT = 19, PART_TOKENS = 8184, MOST_PARTS = 32, MOST_WORKGROUPS = 128;
static_assert(PART_TOKENS < 1 << (32 - PART_SHIFT) && PART_TOKENS << PART_FRACTION < 1 << PART_SHIFT);

template <int TYPE> __device__ __forceinline__ Slice<TYPE> slice_of(const SampleArgs &a, size_t r, int part)
{
    const int size = ((a.vocab + a.parts - 1) / a.parts + 7) / 8 * 8, first = min(part * size, a.vocab);
    return {static_cast<const real_t<TYPE> *>(a.logits) + r * (size_t)a.stride, first, min(first + size, a.vocab)};
}
__device__ __forceinline__ float joined_top(const SampleArgs &a, const Part *parts)
{
    float top = -__builtin_inff();
    bool bad = false;
    for (int i = 0; i < a.parts; ++i) {
        const float t = parts[i].top;
        bad |= t != t;
        top = fmaxf(top, t);
    }
    return bad ? __builtin_nanf("") : top;
}
// a row that has more than one token to draw from
__device__ __forceinline__ bool is_open(const Settings &set, float top) { return !set.bad && top > -__builtin_inff() && !set.first_only(); }

template <int TYPE> __global__ __launch_bounds__(1024) void sample_top_kernel(SampleArgs a)
{
    __shared__ Tops s;
    const size_t r = blockIdx.y;
    const float top = top_of(s, slice_of<TYPE>(a, r, blockIdx.x));
    if (threadIdx.x == 0) (reinterpret_cast<Part *>(a.work) + r * a.parts)[blockIdx.x].top = top;
}

template <int TYPE> __global__ __launch_bounds__(1024) void sample_count_kernel(SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Shared &s = *reinterpret_cast<Shared *>(lds);
    const size_t r = blockIdx.y;
    Part *parts = reinterpret_cast<Part *>(a.work) + r * a.parts;
    const Settings set(a, r);
    const float top = joined_top(a, parts);
    if (!is_open(set, top)) return;
    count_bins(s, slice_of<TYPE>(a, r, blockIdx.x), weigher(a, s, set, top), PART_FRACTION);
    for (int i = threadIdx.x; i < BINS; i += blockDim.x) parts[blockIdx.x].bins[i] = (uint32_t)(s.mass[i] >> 34) << PART_SHIFT | (uint32_t)(s.mass[i] & ((1u << PART_SHIFT) - 1));
}

template <int TYPE> __global__ __launch_bounds__(1024) void sample_weigh_kernel(SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Shared &s = *reinterpret_cast<Shared *>(lds);
    const size_t r = blockIdx.y;
    Part *parts = reinterpret_cast<Part *>(a.work) + r * a.parts, &part = parts[blockIdx.x];
    const Settings set(a, r);
    const float top = joined_top(a, parts);
    if (!is_open(set, top)) return;
    make_table(s);
    // the bins of all parts: four of them per thread
    for (int i = 4 * threadIdx.x; i < BINS; i += 4 * blockDim.x) {
        uint64_t sum[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int p = 0; p < a.parts; ++p) {
            const uint4 v = *reinterpret_cast<const uint4 *>(parts[p].bins + i);
            const uint32_t of[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += (uint64_t)(of[j] >> PART_SHIFT) << 34 | (of[j] & ((1u << PART_SHIFT) - 1));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s.mass[i + j] = sum[j];
    }
    __syncthreads();
    add_up<true>(s, PART_FRACTION);
    make_plan(s, set, PART_FRACTION);
    const Slice<TYPE> slice = slice_of<TYPE>(a, r, blockIdx.x);
    const Weigh w = weigher(a, s, set, top);
    if (s.plan.how == LIST_ALL) list_all(s, slice, w);
    else if (s.plan.how == LIST_ENDS) weigh(s, slice, w, set);
    else start_list(s);
    const uint32_t n = min(s.listed, (uint32_t)LIST);
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        part.list_key[i] = s.list_key[i];
        part.list_mass[i] = s.list_mass[i];
    }
    if (threadIdx.x < SUMS) part.sums[threadIdx.x] = s.sums[threadIdx.x];
    if (threadIdx.x == 0) {
        part.listed = s.listed;
        part.seen = s.count[BINS];
        part.plan = s.plan;
    }
}

template <int TYPE> __global__ __launch_bounds__(1024) void sample_draw_kernel(SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Shared &s = *reinterpret_cast<Shared *>(lds);
    const size_t r = blockIdx.x;
    const Part *parts = reinterpret_cast<const Part *>(a.work) + r * a.parts;
    const Slice<TYPE> row{static_cast<const real_t<TYPE> *>(a.logits) + r * (size_t)a.stride, 0, a.vocab};
    const Settings set(a, r);
    const float top = joined_top(a, parts);
    if (simple_row(a, s, row, set, top, r)) return;
    make_table(s);
    start_list(s);
    // a wave copies the list of a part behind those of the parts before
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (int p = 0; p < a.parts; ++p) {
        const uint32_t n = parts[p].listed;
        if (p % 16 == wave && before + n <= LIST)
            for (uint32_t i = lane; i < n; i += 64) {
                s.list_key[before + i] = parts[p].list_key[i];
                s.list_mass[before + i] = parts[p].list_mass[i];
            }
        before = min(before + n, (uint32_t)(LIST + 1));
    }
    if (threadIdx.x < SUMS)
        for (int p = 0; p < a.parts; ++p) s.sums[threadIdx.x] += parts[p].sums[threadIdx.x];
    if (threadIdx.x == 0) {
        s.listed = before;
        s.plan = parts[0].plan;
    }
    __syncthreads();
    draw(a, s, row, weigher(a, s, set, top), set, parts[0].seen, r);
}

// Parts of a row (1: a row per workgroup): of 8000 tokens or so, for few rows of long vocabularies.  A workgroup takes 0.55 us for 1000 tokens that are all weighed, its parts
// 4 launches.  In one and in parts: 1 x 128000 bfloat16 83 and 48 us, 8 x 128000 95 and 64, 16 x 64000 54 and 50, 1 x 32000 34 and 34, 64 x 64000 63 and 77.
// With top_k few are weighed: 40 and 43, 41 and 45, 29 and 37, 21 and 29.
int row_parts(int rows, int vocab, bool top_k)
{
    const int parts = (vocab + PART_TOKENS - 1) / PART_TOKENS;
    return top_k || parts < 6 || parts > MOST_PARTS || (long long)rows * parts > MOST_WORKGROUPS ? 1 : parts;
}

}  // namespace

size_t sample_workspace_bytes(int rows, int vocab)
{
    // (the most of any number of rows up to this one)
    const int parts = row_parts(1, vocab, false);
    return parts > 1 ? (size_t)std::min(rows, MOST_WORKGROUPS / parts) * parts * sizeof(Part) : 0;
}
bool sample_needs(int rows, int vocab, bool top_k) { return row_parts(rows, vocab, top_k) > 1; }

xnor_status launch_sample(const void *logits, long long stride, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                          const float *uniform, int32_t *token, float *logprob, int32_t *kept, void *workspace, int rows, int vocab, int type, hipStream_t stream)
{
    int b = 0;
    while ((1ll << b) < vocab) ++b;
    const SampleArgs a{logits, temperature, top_p, min_p, uniform, top_k, token, kept, logprob, static_cast<uint8_t *>(workspace), stride, rows, vocab,
                       b > 18 ? 62 - b : 44, b <= 22 ? 12 : 34 - b, row_parts(rows, vocab, top_k != nullptr)};
    xnor_status status = XNOR_OK;
    auto launch = [&](auto kernel, dim3 grid, int threads) {
        if (status) return;
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shared)) != hipSuccess) {
            status = XNOR_ERR_HIP;
            return;
        }
        kernel<<<grid, dim3((unsigned)threads), sizeof(Shared), stream>>>(a);
        status = hip_status(hipGetLastError());
    };
    by_type(type, [&](auto t) {
        if (a.parts == 1) {
            launch(sample_kernel<t()>, dim3((unsigned)rows), vocab > 512 ? 1024 : 256);
            return;
        }
        const dim3 all((unsigned)a.parts, (unsigned)rows);
        sample_top_kernel<t()><<<all, dim3(1024), 0, stream>>>(a);
        status = hip_status(hipGetLastError());
        launch(sample_count_kernel<t()>, all, 1024);
        launch(sample_weigh_kernel<t()>, all, 1024);
        launch(sample_draw_kernel<t()>, dim3((unsigned)rows), 1024);
    });
    return status;
}

}  // namespace xnor
