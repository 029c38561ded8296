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

// 2^(i / 256)
struct Powers {
    double of[PER_OCTAVE];
    constexpr Powers() : of()
    {
        for (int i = 0; i < PER_OCTAVE; ++i) {
            const double x = i * (0x1.62e42fefa39efp-1 / PER_OCTAVE);
            double sum = 0.0;
            for (int k = 24; k > 0; --k) sum = (sum + 1.0) * (x / k);          // e^x - 1 by its series, the smallest terms first
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
    float part, part_top, bin_factor;
    double top, factor, whole;
    const double *table;            // 2^(i / 256)
    __device__ __forceinline__ Weigh(float largest, float T, int bits, const double *powers)
    {
        // temperatures near the ends of float32 weigh logits as close together, if these are small themselves (others are 2^75 temperatures apart, or the same)
        const bool close = T < 0x1p-100f && __builtin_fabsf(largest) < 1.0f;
        part = close ? 0x1p60f : 0.5f;
        part_top = part * largest;
        bin_factor = fminf(PER_E / (part * T), 0x1.fffffep127f);
        top = largest;
        factor = PER_OCTAVE * 0x1.71547652b82fep+0 / (double)T;                // log2 e
        whole = 0x1.8p52 + PER_OCTAVE * bits;
        table = powers;
    }
    // in bins, as a real number: in 32 bits, where it never falls as the logit falls (both roundings keep the order), and that is all a bin has to do.  (From the halves: the
    // distance itself may be out of range.)
    __device__ __forceinline__ float bins(float l) const { return __builtin_fmaf(l, -part, part_top) * bin_factor; }
    __device__ __forceinline__ static int bin(float b) { return (int)fminf(b, BINS - 1); }
    // in 256ths of a factor of two
    __device__ __forceinline__ double distance(float l) const { return (top - (double)l) * factor; }
    // 2^bits exp(-distance), rounded to a whole number, for a distance below NO_WEIGHT.  Rounding and scaling by additions: their own instructions take four times as long.
    __device__ __forceinline__ double weight(float l) const
    {
        constexpr double c = 0x1.62e42fefa39efp-9;                              // ln 2 / 256
        const double d = (double)l - top, n = __builtin_fma(d, factor, whole), x = __builtin_fma(d, factor, whole - n);
        const double e = __builtin_fma(x, __builtin_fma(x, __builtin_fma(x, c * c * c / 6, c * c / 2), c), 1.0);          // (the next term: 1.4e-13 at most)
        const int i = (int)(uint32_t)__builtin_bit_cast(uint64_t, n);           // 256 bits - the whole 256ths
        const uint64_t w = __builtin_bit_cast(uint64_t, table[i & (PER_OCTAVE - 1)] * e);
        const uint32_t high = (uint32_t)(w >> 32) + ((uint32_t)(i & -PER_OCTAVE) << 12);
        return (__builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)w) + 0x1p52) - 0x1p52;
    }
    // (weights are 2^44 at most: the digits behind 2^52)
    static __device__ __forceinline__ uint64_t digits(double weight) { return __builtin_bit_cast(uint64_t, weight + 0x1p52) & 0xfffffffffffffull; }
    __device__ __forceinline__ uint64_t whole_weight(float l) const { return distance(l) < NO_WEIGHT ? digits(weight(l)) : 0; }
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
    uint32_t wave_tokens[16];
    uint32_t listed;
    int first[6], found_bin;
    uint64_t found_before_mass, found_before_count;
    Plan plan;
};

// What the tokens up to some place in the order amount to, that one with them.
struct Place {
    uint64_t count, mass, key;
};

// Sums over the lanes up to this one: of 16 neighbours (WIDTH 16) or of the wave, without a way through LDS.
template <int WIDTH, class T> __device__ __forceinline__ T lanes_upto(T v)
{
    // (lanes whose source is outside of their row, or whose row is masked, add 0)
    const auto step = [&](auto control, auto rows) {
        constexpr int C = decltype(control)::value, R = decltype(rows)::value;
        if constexpr (sizeof(T) == 8) {
            const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, C, R, 0xf, false);
            const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)v >> 32), C, R, 0xf, false);
            v += (uint64_t)high << 32 | low;
        } else {
            v += (T)__builtin_amdgcn_update_dpp(0, (int)v, C, R, 0xf, false);
        }
    };
    step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());        // 1, 2, 4 and 8 lanes to the right
    step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
    if constexpr (WIDTH == 64) {
        step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());    // a row's last lane to the next row (rows 1 and 3), lane 31 to the upper half
        step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
    }
    return v;
}
template <class T> __device__ __forceinline__ T lane_of(T v, int lane)
{
    if constexpr (sizeof(T) == 8)
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
    else return (T)__builtin_amdgcn_readlane((int)v, lane);
}
// What the waves before this one have in their slots, and what all have.
template <class T> __device__ __forceinline__ T waves_before(const T *slots, T &all)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const T upto = lanes_upto<16>((lane & 15) < waves ? slots[lane & 15] : (T)0);
    all = lane_of(upto, 15);
    return wave ? lane_of(upto, wave - 1) : (T)0;
}
// Sum over the threads before this one, and over all.
__device__ __forceinline__ uint64_t scan(uint64_t v, uint64_t *slots, uint64_t &all)
{
    const uint64_t upto = lanes_upto<64>(v);
    if ((threadIdx.x & 63) == 63) slots[threadIdx.x >> 6] = upto;
    __syncthreads();
    const uint64_t before = waves_before(slots, all);
    __syncthreads();
    return before + upto - v;
}

// A row's tokens first .. last - 1.
template <int TYPE> struct Slice {
    typedef real_t<TYPE> T;
    const T *l;
    int first, last;
    // f(eight of them, the first one's index), -inf behind the end; the next eight are on their way meanwhile
    template <class F> __device__ __forceinline__ void eights(F f) const
    {
        const int step = 8 * blockDim.x;
        auto load = [&](int c) {
            Real8<TYPE> v;
            if (c < last) v.load(l + c, last - c, -__builtin_inff());
            return v;
        };
        int c = first + 8 * (int)threadIdx.x;
        Real8<TYPE> next = load(c);
        for (; c < last; c += step) {
            const Real8<TYPE> v = next;
            next = load(c + step);
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
    if (a.logprob) a.logprob[r] = fminf((float)(((double)logit_of(key) - w.top) / (double)T - log(__builtin_ldexp((double)mass, -a.bits))), 0.0f);
}

__device__ __forceinline__ void make_table(Shared &s)
{
    for (int i = threadIdx.x; i < PER_OCTAVE; i += blockDim.x) s.table[i] = powers.of[i];
}

// Into s.mass: the count in the upper 30 bits, the sum of the distances within the bin in the 34 below.  (2^30 tokens in one bin, all there can be, would count as none: the plan then
// lists everything, which does not fit, and the ends are looked for.)
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
// What a bin's counts and distances stand for: weights in 2^-32, at the mean distance of its tokens (their mean weight is above that by 1 / (8 * 128^2) at most).  All in 32 bits.
__device__ __forceinline__ uint64_t estimate(uint64_t counted, int bin, float step)
{
    const float n = (float)(uint32_t)(counted >> 34);
    const float sum = __builtin_fmaf((float)((uint32_t)(counted >> 32) & 3u), 0x1p32f, (float)(uint32_t)counted);
    const float within = __builtin_fmaf(sum, __builtin_amdgcn_rcpf(n), 0.5f) * step;
    const float mass = fmaxf(n * __builtin_amdgcn_exp2f(((float)bin + within) * (-1.44269504f / PER_E)) * 0x1p32f, 1.0f);          // (a bin that holds any ends somewhere)
    const uint32_t high = (uint32_t)(mass * 0x1p-32f), low = (uint32_t)__builtin_fmaf((float)high, -0x1p32f, mass);
    return n > 0.0f ? (uint64_t)high << 32 | low : 0;
}

// The bins' counts and masses become those of all before.  COUNTED: s.mass holds what count_bins left.
template <bool COUNTED> __device__ __forceinline__ void add_up(Shared &s, int fraction)
{
    constexpr int PER = 4;
    const float step = COUNTED ? 1.0f / (float)(1 << fraction) : 0.0f;
    uint32_t base_c = 0;
    uint64_t base_m = 0;
    for (int first = 0; first < BINS; first += PER * blockDim.x) {          // (once, with 1024 threads)
        const int at = first + PER * threadIdx.x;
        uint32_t c[PER], own_c = 0;
        uint64_t m[PER], own_m = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            m[i] = s.mass[at + i];
            c[i] = COUNTED ? (uint32_t)(m[i] >> 34) : s.count[at + i];
            if (COUNTED) m[i] = estimate(m[i], at + i, step);
            own_c += c[i];
            own_m += m[i];
        }
        const uint32_t upto_c = lanes_upto<64>(own_c);
        const uint64_t upto_m = lanes_upto<64>(own_m);
        if ((threadIdx.x & 63) == 63) {
            s.wave_tokens[threadIdx.x >> 6] = upto_c;
            s.wave_mass[threadIdx.x >> 6] = upto_m;
        }
        __syncthreads();
        uint32_t all_c;
        uint64_t all_m;
        uint32_t before_c = base_c + waves_before(s.wave_tokens, all_c) + upto_c - own_c;
        uint64_t before_m = base_m + waves_before(s.wave_mass, all_m) + upto_m - own_m;
        base_c += all_c;
        base_m += all_m;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s.count[at + i] = before_c;
            s.mass[at + i] = before_m;
            before_c += c[i];
            before_m += m[i];
        }
        if (first + PER * (int)blockDim.x >= BINS && threadIdx.x == 0) {
            s.count[BINS] = base_c;
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

// The same by a whole wave: 64 places at a time.
template <class T> __device__ __forceinline__ int bin_of_wide(const T *before, T target)
{
    static_assert(BINS == 64 * 64);
    const int lane = threadIdx.x & 63;
    const int block = max((int)__popcll(__ballot(before[64 * lane] < target)) - 1, 0);
    return 64 * block + max((int)__popcll(__ballot(before[64 * block + lane] < target)) - 1, 0);
}

// In 256ths of a factor of two, the distance of weight min_p.
__device__ __forceinline__ double furthest_of(const Settings &set)
{
    return set.min_p > 0.0f ? fmax(-PER_OCTAVE * log2((double)set.min_p), 0.0) : __builtin_inf();
}

__device__ __forceinline__ int list_size() { return min(LIST, (int)blockDim.x); }        // (sorted by a thread each)

// From the counts and the estimated masses.  An estimate is within 1.2e-5 of the true mass (the mean distance 8e-6, float32 the rest) and half a step of the distances, so that
// a share of the whole lies within twice that of where the estimates put it.
__device__ __forceinline__ void make_plan(Shared &s, const Settings &set, int fraction)
{
    if (threadIdx.x < 64) {
        const double width = 2.4 * (1.2e-5 + 0.5 / PER_E / (1 << fraction));
        Plan p;
        p.p_first = BINS;                   // (none)
        p.p_last = p.k_first = -1;
        p.last = BINS - 1;
        p.k_before = p.p_before = 0;
        uint64_t least = s.mass[BINS], most = least;
        uint32_t wanted = 0;
        auto look = [&](double share, int &first, int &last, uint32_t &before) {
            first = min(bin_of_wide(s.mass, (uint64_t)fmin(fmax(share * (double)least * (1 - width), 1.0), (double)most)), p.last);
            last = min(bin_of_wide(s.mass, (uint64_t)fmin(fmax(share * (double)most * (1 + width), 1.0), (double)most)), p.last);
            before = s.count[first];
            wanted += s.count[last + 1] - before;
        };
        if (set.top_k > 0 && (uint32_t)set.top_k < s.count[BINS]) {
            p.last = p.k_first = bin_of_wide(s.count, (uint32_t)set.top_k);
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
        // (more than half a list takes the long sort, 10 us: 1 x 1000 float32 26 us, by its ends 14)
        const uint32_t fits = (uint32_t)list_size(), all = s.count[p.last + 1];
        p.how = all <= fits / 2 ? LIST_ALL : wanted <= fits / 2 ? LIST_ENDS : all <= fits ? LIST_ALL : wanted <= fits ? LIST_ENDS : SEARCH;
        if (threadIdx.x == 0) s.plan = p;
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
// What bounds it: vector instructions, about 40 for a token, half of them of 64 bits (256 x 32000: 12 us).
template <int TYPE> __device__ __forceinline__ void weigh(Shared &s, const Slice<TYPE> &slice, const Weigh &w, const Settings &set)
{
    const Plan p = s.plan;
    start_list(s);
    const bool by_count = p.k_first >= 0, by_mass = p.p_first <= p.p_last, by_weight = set.min_p > 0.0f;
    const double furthest = furthest_of(set);
    // bins as real numbers: what is in bin i lies from i to below i + 1, in the last one from there on.  (A masked token is at an infinity or NaN, in none of them.)
    const auto end = [](int bin) { return bin < BINS - 1 ? (float)(bin + 1) : __builtin_inff(); };
    const float last = end(p.last), weighed = fminf(last, BINS - 1);           // (what is behind weighs nothing: where it is listed, a 0)
    const float k_first = by_count ? (float)p.k_first : __builtin_inff(), p_first = by_mass ? (float)p.p_first : __builtin_inff(), u_first = (float)p.u_first;
    const float p_end = end(p.p_last), u_end = end(p.u_last);
    double sum_k = 0, sum_p = 0, sum_u = 0, sum_min = 0;
    uint32_t count_min = 0;
    const auto pass = [&](auto count, auto mass, auto weight) {
        slice.eights([&](const Real8<TYPE> &v, int c) {
#pragma unroll
            for (int pair = 0; pair < 4; ++pair) {              // (two at a time: more of them side by side leave no registers)
                bool listed[2];
                double m[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float l = v[2 * pair + j], b = w.bins(l);
                    m[j] = w.weight(l);
                    m[j] = b < weighed ? m[j] : 0.0;
                    sum_k = count() ? __builtin_fma(m[j], b < k_first ? 1.0 : 0.0, sum_k) : sum_k + m[j];
                    if (mass()) sum_p = __builtin_fma(m[j], b < p_first ? 1.0 : 0.0, sum_p);
                    sum_u = __builtin_fma(m[j], b < u_first ? 1.0 : 0.0, sum_u);
                    if (weight()) {
                        const bool is = (b < last) & (w.distance(l) <= furthest);
                        sum_min = __builtin_fma(m[j], is ? 1.0 : 0.0, sum_min);
                        count_min += is;
                    }
                    listed[j] = (b >= u_first) & (b < u_end);
                    if (mass()) listed[j] |= (b >= p_first) & (b < p_end);
                    if (count()) listed[j] |= (b >= k_first) & (b < last);          // (top_k's bin is the last one)
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (listed[j]) {
                        uint32_t at;
                        if (put(s, v[2 * pair + j], c + 2 * pair + j, at)) s.list_mass[at] = Weigh::digits(m[j]);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    };
    // (each end that is not asked for saves 3 instructions of some 35 for a token)
    typedef std::true_type yes;
    typedef std::false_type no;
    if (by_weight) pass(yes(), yes(), yes());
    else if (by_count) by_mass ? pass(yes(), yes(), no()) : pass(yes(), no(), no());
    else by_mass ? pass(no(), yes(), no()) : pass(no(), no(), no());
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

constexpr int FEW = 256;            // listed tokens that one wave takes, without waiting for the others: 2 us less than with all of them for 100

// A list in order: s.list_key, and in s.list_mass the weights of the listed ones up to each.
// Few: the first wave alone, four tokens per lane; otherwise all waves, one per thread.
template <bool WEIGHED> __device__ __forceinline__ void sort_long(Shared &s, int n)
{
    const int i = threadIdx.x;
    uint64_t key = i < n ? s.list_key[i] : ~0ull, own = WEIGHED && i < n ? s.list_mass[i] : 0;
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
    __syncthreads();
    s.list_key[i] = key;
    if (WEIGHED) s.list_mass[i] = own;
}
template <bool WEIGHED> __device__ __forceinline__ void sort(Shared &s, int n)
{
    if (n > (int)blockDim.x / 2) {
        sort_long<WEIGHED>(s, n);
    } else {
        // each token's place by counting those before it, several threads to a token (256 of 1024: 2 us, 512: 7; the sort takes 15)
        int share = 2;
        while (share < 64 && 2 * share * n <= (int)blockDim.x) share *= 2;
        const int of = threadIdx.x / share;
        const uint64_t mine = of < n ? s.list_key[of] : 0, its = WEIGHED && of < n ? s.list_mass[of] : 0;
        int before = 0;
#pragma unroll 4
        for (int j = threadIdx.x & (share - 1); j < n; j += share) before += s.list_key[j] < mine;
        for (int d = share / 2; d > 0; d >>= 1) before += __shfl_xor(before, d, 64);
        __syncthreads();
        if (of < n && (threadIdx.x & (share - 1)) == 0) {
            s.list_key[before] = mine;
            if (WEIGHED) s.list_mass[before] = its;
        }
    }
    __syncthreads();
}
template <bool IS_FEW> struct Listed {
    static constexpr int PER = IS_FEW ? FEW / 64 : 1;
    uint64_t key[PER], upto[PER];
    int first_index;
    // (IS_FEW: of a list in order, in the first wave)
    template <bool WEIGHED> static __device__ __forceinline__ Listed make(Shared &s, const Weigh &w, int n)
    {
        Listed l;
        l.first_index = PER * (int)threadIdx.x;
        uint64_t all = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = l.first_index + k;
            l.key[k] = i < n ? s.list_key[i] : ~0ull;
            all += i >= n ? 0 : WEIGHED ? s.list_mass[i] : w.whole_weight(logit_of(l.key[k]));
            l.upto[k] = all;
        }
        uint64_t whole;
        const uint64_t before = IS_FEW ? lanes_upto<64>(all) - all : scan(all, s.wave_mass, whole);
#pragma unroll
        for (int k = 0; k < PER; ++k) s.list_mass[l.first_index + k] = l.upto[k] += before;
        wait();
        return l;
    }
    static __device__ __forceinline__ void wait()
    {
        if (IS_FEW) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");          // (what a wave writes to LDS it reads in order)
        else __syncthreads();
    }
    // The first one of which f(its index, key, weights up to it) is true, LIST if none; `slot` of s.first holds LIST before.
    template <class F> __device__ __forceinline__ int first(Shared &s, int slot, F f) const
    {
        if constexpr (IS_FEW) {
            int mine = LIST;
#pragma unroll
            for (int k = PER - 1; k >= 0; --k) mine = f(first_index + k, key[k], upto[k]) ? first_index + k : mine;
            const uint64_t any = __ballot(mine < LIST);
            return any ? __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(any)) : LIST;
        } else {
            const uint64_t all = __ballot(f(first_index, key[0], upto[0]));
            if (all && (threadIdx.x & 63) == 0) atomicMin(&s.first[slot], (int)threadIdx.x + __builtin_ctzll(all));
            __syncthreads();
            return s.first[slot];
        }
    }
};

// From a list in order of all tokens that count.
template <bool IS_FEW> __device__ __forceinline__ void draw_listed(const SampleArgs &a, Shared &s, const Weigh &w, const Settings &set, uint32_t seen, size_t r, int n)
{
    const Listed<IS_FEW> l = Listed<IS_FEW>::template make<false>(s, w, n);
    int count = set.top_k > 0 && (uint32_t)set.top_k < seen ? set.top_k : (int)seen;
    uint64_t mass = s.list_mass[count - 1];
    if (set.top_p < 1.0f) {
        const uint64_t target = set.top_target(mass);
        count = l.first(s, 0, [&](int i, uint64_t, uint64_t upto) { return i < count && upto >= target; }) + 1;
    }
    if (set.min_p > 0.0f) {
        const double furthest = furthest_of(set);
        count = min(count, l.first(s, 1, [&](int i, uint64_t key, uint64_t) { return i >= n || w.distance(logit_of(key)) > furthest; }));
    }
    mass = s.list_mass[count - 1];
    const uint64_t target = set.draw_target(mass);
    const int at = l.first(s, 2, [&](int, uint64_t, uint64_t upto) { return upto >= target; });
    if (threadIdx.x == 0) write_drawn(a, w, set.T, r, s.list_key[at], count, mass);
}
// False: the list is too short.
__device__ __forceinline__ bool draw_all(const SampleArgs &a, Shared &s, const Weigh &w, const Settings &set, uint32_t seen, size_t r)
{
    const int n = (int)min(s.listed, (uint32_t)LIST + 1);
    if (n > list_size()) return false;
    sort<false>(s, n);
    if (n > FEW) draw_listed<false>(a, s, w, set, seen, r, n);
    else if (threadIdx.x < 64) draw_listed<true>(a, s, w, set, seen, r, n);
    return true;
}

// From the sums and the list in order.  False: the plan did not hold what was looked for.
template <bool IS_FEW> __device__ __forceinline__ bool draw_between(const SampleArgs &a, Shared &s, const Weigh &w, const Settings &set, uint32_t seen, size_t r, int n)
{
    const Plan plan = s.plan;
    const Listed<IS_FEW> l = Listed<IS_FEW>::template make<true>(s, w, n);
    const bool by_count = plan.k_first >= 0, by_mass = plan.p_first <= plan.p_last;
    uint64_t count = seen, mass = s.sums[SUM_K];
    const auto bin = [&](int i, uint64_t key) { return i < n ? Weigh::bin(w.bins(logit_of(key))) : BINS; };
    const auto start_of = [&](int slot, int first) { return l.first(s, slot, [&](int i, uint64_t key, uint64_t) { return bin(i, key) >= first; }); };
    // what the listed ones before a bin's first weigh
    const auto before = [&](int first) { return first > 0 ? s.list_mass[min(first, n) - 1] : 0; };
    if (by_count) {
        const int start = start_of(0, plan.k_first), at = start + (int)(set.top_k - plan.k_before) - 1;
        if (at >= n) return false;
        count = set.top_k;
        mass += s.list_mass[at] - before(start);
    }
    if (by_mass) {
        const int start = start_of(1, plan.p_first);
        const uint64_t base = s.sums[SUM_P] - before(start), target = set.top_target(mass);
        const int at = l.first(s, 2, [&](int i, uint64_t key, uint64_t upto) {
            const int b = bin(i, key);
            return b >= plan.p_first && b <= plan.p_last && base + upto >= target;
        });
        if (at >= n || s.sums[SUM_P] >= target) return false;
        count = plan.p_before + (at - start) + 1;
        mass = base + s.list_mass[at];
    }
    if (set.min_p > 0.0f) {
        count = min((unsigned long long)count, (unsigned long long)s.sums[COUNT_MIN]);
        mass = min((unsigned long long)mass, (unsigned long long)s.sums[SUM_MIN]);
    }
    const int start = start_of(3, plan.u_first);
    const uint64_t base = s.sums[SUM_U] - before(start), target = set.draw_target(mass);
    const int at = l.first(s, 4, [&](int i, uint64_t key, uint64_t upto) {
        const int b = bin(i, key);
        return b >= plan.u_first && b <= plan.u_last && base + upto >= target;
    });
    if (at >= n || s.sums[SUM_U] >= target) return false;
    if (threadIdx.x == 0) write_drawn(a, w, set.T, r, s.list_key[at], count, mass);
    return true;
}
// False: that, or the list is too short.
__device__ __forceinline__ bool draw_ends(const SampleArgs &a, Shared &s, const Weigh &w, const Settings &set, uint32_t seen, size_t r)
{
    const int n = (int)min(s.listed, (uint32_t)LIST + 1);
    if (n > list_size()) return false;
    sort<true>(s, n);
    if (n > FEW) return draw_between<false>(a, s, w, set, seen, r, n);
    if (threadIdx.x < 64) {
        const bool drawn = draw_between<true>(a, s, w, set, seen, r, n);
        if (threadIdx.x == 0) s.found_bin = drawn;
    }
    __syncthreads();
    return s.found_bin != 0;
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
    const int n = (int)s.listed;
    sort<false>(s, n);
    const Listed<false> l = Listed<false>::make<false>(s, w, n);
    const uint64_t rest = target - (BY_MASS ? before_mass : before_count);
    const int at = l.first(s, 0, [&](int i, uint64_t, uint64_t upto) { return (BY_MASS ? upto : (uint64_t)i + 1) >= rest; });
    const Place p{before_count + at + 1, before_mass + s.list_mass[at], s.list_key[at]};
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
    return Weigh(top, set.T, a.bits, s.table);
}

// From what a pass over the whole row left.
template <int TYPE> __device__ __forceinline__ void draw(const SampleArgs &a, Shared &s, const Slice<TYPE> &row, const Weigh &w, const Settings &set, uint32_t seen, size_t r)
{
    if (s.plan.how == LIST_ALL && draw_all(a, s, w, set, seen, r)) return;
    if (s.plan.how == LIST_ENDS && draw_ends(a, s, w, set, seen, r)) return;
    draw_searched(a, s, row, w, set, r);
}

// A row per workgroup.
// What bounds it: the row's CU, most of all its vector instructions: 256 x 32000 bfloat16 with top_p 26 us, of which 4 read the row, 4 count it (atomics in LDS), 12 weigh all
// tokens, 3 list and draw, the rest adds up the bins and starts; with min_p too 29, with a top_k of 64 17, settings of each row 30 to 32.  Rows that their ends are looked for in by
// themselves: 91 where the logits are nearly flat (deviation 0.05), 690 where all are alike; one of 128000 in parts 270 and 1360.
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
    uint32_t bins[BINS];            // count in the upper 13 bits, the mean distance within the bin in the 19 below
    uint64_t list_key[LIST], list_mass[LIST], sums[SUMS];
    float top;
    uint32_t listed, seen;          // seen, plan: of the first part only, for the row
    Plan plan;
};
constexpr int PART_FRACTION = 12, MEAN_BITS = 19, PART_TOKENS = 8184, MOST_PARTS = 64, MOST_WORKGROUPS = 256;
static_assert(PART_TOKENS < 1 << (32 - MEAN_BITS) && (uint64_t)MOST_PARTS * PART_TOKENS << PART_FRACTION < 1ull << 32);

template <int TYPE> __device__ __forceinline__ Slice<TYPE> slice_of(const SampleArgs &a, size_t r, int part)
{
    const int size = ((a.vocab + a.parts - 1) / a.parts + 7) / 8 * 8, first = min(part * size, a.vocab);
    return {static_cast<const real_t<TYPE> *>(a.logits) + r * (size_t)a.stride, first, min(first + size, a.vocab)};
}
__device__ __forceinline__ float joined_top(const SampleArgs &a, const Part *parts)
{
    // (a lane for each part: one after another they cost the way to memory each)
    float top = parts[min((int)(threadIdx.x & 63), a.parts - 1)].top;
    const bool bad = __any(top != top);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
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
    for (int i = threadIdx.x; i < BINS; i += blockDim.x) {
        const uint32_t n = (uint32_t)(s.mass[i] >> 34);
        const float mean = (float)(uint32_t)s.mass[i] / (float)max(n, 1u);             // (a part's sums are below 2^32)
        const uint32_t its = min((uint32_t)(mean * (1 << (MEAN_BITS - PART_FRACTION)) + 0.5f), (1u << MEAN_BITS) - 1);
        parts[blockIdx.x].bins[i] = n << MEAN_BITS | its;
    }
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
    // the bins of all parts: four of them per thread, eight parts on their way at once
    for (int i = 4 * threadIdx.x; i < BINS; i += 4 * blockDim.x) {
        uint32_t count[4] = {0, 0, 0, 0}, within[4] = {0, 0, 0, 0};
        for (int first = 0; first < a.parts; first += 8) {
            uint4 v[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) v[p] = *reinterpret_cast<const uint4 *>(parts[min(first + p, a.parts - 1)].bins + i);
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                const uint32_t of[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t its = first + p < a.parts ? of[j] : 0;
                    const uint32_t n = its >> MEAN_BITS;
                    count[j] += n;
                    within[j] += n * (its & ((1u << MEAN_BITS) - 1)) >> (MEAN_BITS - PART_FRACTION);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s.mass[i + j] = (uint64_t)count[j] << 34 | within[j];
    }
    __syncthreads();
    add_up<true>(s, PART_FRACTION);
    make_plan(s, set, PART_FRACTION - 1);          // (means and products of them are rounded: another half of a step)
    const Slice<TYPE> slice = slice_of<TYPE>(a, r, blockIdx.x);
    const Weigh w = weigher(a, s, set, top);
    if (s.plan.how == LIST_ALL) list_all(s, slice, w);
    else if (s.plan.how == LIST_ENDS) weigh(s, slice, w, set);
    else start_list(s);
    const uint32_t n = min(s.listed, (uint32_t)LIST);
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        part.list_key[i] = s.list_key[i];
        part.list_mass[i] = s.list_mass[i];             // (of LIST_ALL nothing that is used: to ask for the plan before a list is copied takes 0.7 us of 42, 1 x 262144)
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
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const uint32_t own = lane < a.parts ? min(parts[lane].listed, (uint32_t)(LIST + 1)) : 0, upto = lanes_upto<64>(own);
    for (int p = wave; p < a.parts; p += waves) {
        const uint32_t n = lane_of(own, p), before = lane_of(upto, p) - n;
        if (before + n <= LIST)
            for (uint32_t i = lane; i < n; i += 64) {
                s.list_key[before + i] = parts[p].list_key[i];
                s.list_mass[before + i] = parts[p].list_mass[i];
            }
    }
    if ((int)threadIdx.x < SUMS * a.parts)
        atomicAdd((unsigned long long *)&s.sums[threadIdx.x % SUMS], (unsigned long long)parts[threadIdx.x / SUMS].sums[threadIdx.x % SUMS]);
    if (threadIdx.x == 0) {
        s.listed = lane_of(upto, 63);
        s.plan = parts[0].plan;
    }
    __syncthreads();
    draw(a, s, row, weigher(a, s, set, top), set, parts[0].seen, r);
}

// Parts of a row (1: a row per workgroup): of 8000 tokens or so, for few rows of long vocabularies.  A workgroup takes 0.4 us for 1000 tokens that are all weighed, its parts
// 4 launches.  In one and in parts, with top_p: 1 x 128000 bfloat16 66 and 32 us, 16 x 128000 74 and 45, 1 x 41000 30 and 28, 24 x 64000 42 and 37, 1 x 32000 26 and 28, 32 x 50000
// 35 and 37, 64 x 64000 46 and 66, 1 x 262144 129 and 42, 4 x 523776 250 and 59.  With top_k few are weighed: 40 and 43 (1 x 128000), 29 and 37, 21 and 29.  (No more parts
// than a wave has lanes, which join what they hand on.)
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
