// Tokens drawn from rows of logits by temperature, top-k, top-p and min-p (contract: xnor_lowbit.h).
//
// Nothing is sorted.  The tokens' order (largest logit first, then lowest index) is walked by digits: the first is the logit's distance to the largest one in steps of a
// 32nd of a factor of two of the weight, the others are the bits of (logit, index).  Every search (the last of top_k, the last of top_p, the token drawn) is for the
// first place in that order where a measure (number of tokens, or their weight) reaches a target: a histogram over a digit gives the bin that it is in, and once that
// holds few tokens they are listed and ranked.  The first digit's histogram serves all searches.
//
// Weights are integers: exp(-d / T) in 64 bits, times a power of two, rounded.  Their sums are exact and depend on no order.
#include "xnor_internal.h"
#include "real8.h"
#include "lowbit.h"

namespace xnor {

namespace {

constexpr int BINS = 2048, LIST = 512, PER_OCTAVE = 256, BIN_SHIFT = 3;     // bins of 8 / 256 of a factor of two: 64 factors of two in all
constexpr double NO_WEIGHT = BINS * 8 - 1;          // in 256ths of a factor of two: from there on weights round to 0 (2^-63)

struct SampleArgs {
    const void *logits;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *logprob;
    long long stride;
    int rows, vocab, bits;          // bits of a weight of 1
};

// A row's distances and weights.
struct Weigh {
    double largest, factor;
    int bits;
    const double *table;            // 2^(-i / 256)
    // in 256ths of a factor of two
    __device__ __forceinline__ double distance(float l) const { return fmin((largest - (double)l) * factor, NO_WEIGHT); }
    __device__ __forceinline__ static int bin(double t) { return (int)__builtin_rint(t) >> BIN_SHIFT; }
    __device__ __forceinline__ double weight(double t, int bits) const          // times 2^bits
    {
        const double n = __builtin_rint(t), x = (n - t) * 0x1.62e42fefa39efp-9;          // ln 2 / 256
        const double e = __builtin_fma(x, __builtin_fma(x, __builtin_fma(x, __builtin_fma(x, 1.0 / 24, 1.0 / 6), 0.5), 1.0), 1.0);
        const int i = (int)n;
        return __builtin_ldexp(table[i & 255] * e, bits - (i >> 8));
    }
    __device__ __forceinline__ static uint64_t rounded(double w) { return __builtin_bit_cast(uint64_t, w + 0x1p52) & 0xfffffffffffffull; }
};

// Largest first, of equal ones (0 and -0 among them) the lowest index first.
__device__ __forceinline__ uint64_t key_of(float l, int index)
{
    const uint32_t u = __float_as_uint(l + 0.0f);
    return (uint64_t)~(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)index;
}

struct Shared {
    uint64_t mass[2][BINS];
    uint32_t count[2][BINS];
    double table[256];
    uint64_t list_key[LIST], list_mass[LIST];
    uint64_t wave_mass[16], wave_count[16];
    float wave_top[16];
    int wave_bad[16];
    uint32_t listed;
    int found_bin;
    uint64_t found_before_mass, found_before_count, found_key, found_mass, found_count, found_own;
};

struct Place {          // of a search: what the tokens up to and with the one found amount to
    uint64_t count, mass, key, own;
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

template <int TYPE> struct Row {
    typedef real_t<TYPE> T;
    const T *l;
    int vocab;
    // f(logit, index) for every one above -inf
    template <class F> __device__ __forceinline__ void each(F f) const
    {
        for (int c = 8 * threadIdx.x; c < vocab; c += 8 * blockDim.x) {
            Real8<TYPE> v;
            v.load(l + c, vocab - c, -__builtin_inff());
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v[j] > -__builtin_inff()) f(v[j], c + j);
        }
    }
};

// The bin of a histogram where the measure, on top of what lies before, reaches the target.
__device__ __forceinline__ void find_bin(Shared &s, int h, bool by_mass, uint64_t target, uint64_t before_count, uint64_t before_mass)
{
    const int per = BINS / blockDim.x, first = threadIdx.x * per;
    uint64_t c = 0, m = 0, all;
    for (int i = 0; i < per; ++i) {
        c += s.count[h][first + i];
        m += s.mass[h][first + i];
    }
    uint64_t bc = before_count + scan(c, s.wave_count, all), bm = before_mass + scan(m, s.wave_mass, all);
    const uint64_t start = by_mass ? bm : bc;
    if (start < target && target <= start + (by_mass ? m : c))
        for (int i = 0; i < per; ++i) {
            const uint64_t nc = bc + s.count[h][first + i], nm = bm + s.mass[h][first + i];
            if ((by_mass ? nm : nc) >= target) {
                s.found_bin = first + i;
                s.found_before_count = bc;
                s.found_before_mass = bm;
                break;
            }
            bc = nc;
            bm = nm;
        }
    __syncthreads();
}

// The first place in the order where the measure reaches the target (1 .. all of it).
template <int TYPE> __device__ Place search(Shared &s, const Row<TYPE> &row, const Weigh &w, bool by_mass, uint64_t target)
{
    find_bin(s, 0, by_mass, target, 0, 0);
    const int bin0 = s.found_bin;
    uint64_t before_count = s.found_before_count, before_mass = s.found_before_mass, prefix = 0, mask = 0;
    uint32_t in_bin = s.count[0][bin0];
    int shift = 64;
    while (in_bin > LIST) {         // (ends: the keys differ, and the last digit is 9 bits)
        const int next = shift > 11 ? shift - 11 : 0, width = shift - next;
        __syncthreads();
        for (int i = threadIdx.x; i < BINS; i += blockDim.x) {
            s.count[1][i] = 0;
            s.mass[1][i] = 0;
        }
        __syncthreads();
        row.each([&](float l, int index) {
            const double t = w.distance(l);
            const uint64_t key = key_of(l, index);
            if (Weigh::bin(t) != bin0 || (key & mask) != prefix) return;
            const int d = (int)(key >> next) & ((1 << width) - 1);
            atomicAdd(&s.count[1][d], 1u);
            atomicAdd((unsigned long long *)&s.mass[1][d], (unsigned long long)Weigh::rounded(w.weight(t, w.bits)));
        });
        __syncthreads();
        find_bin(s, 1, by_mass, target, before_count, before_mass);
        before_count = s.found_before_count;
        before_mass = s.found_before_mass;
        prefix |= (uint64_t)s.found_bin << next;
        mask |= (uint64_t)((1u << width) - 1) << next;
        in_bin = s.count[1][s.found_bin];
        shift = next;
    }
    __syncthreads();
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    row.each([&](float l, int index) {
        const double t = w.distance(l);
        const uint64_t key = key_of(l, index);
        if (Weigh::bin(t) != bin0 || (key & mask) != prefix) return;
        const uint32_t at = atomicAdd(&s.listed, 1u);
        if (at < LIST) {
            s.list_key[at] = key;
            s.list_mass[at] = Weigh::rounded(w.weight(t, w.bits));
        }
    });
    __syncthreads();
    const int n = min((int)s.listed, LIST);
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const uint64_t key = s.list_key[i], own = s.list_mass[i];
        uint64_t c = before_count + 1, m = before_mass + own;
        for (int j = 0; j < n; ++j)
            if (s.list_key[j] < key) {
                ++c;
                m += s.list_mass[j];
            }
        const uint64_t here = by_mass ? m : c, step = by_mass ? own : 1;
        if (here >= target && here - step < target) {
            s.found_key = key;
            s.found_count = c;
            s.found_mass = m;
            s.found_own = own;
        }
    }
    __syncthreads();
    const Place p{s.found_count, s.found_mass, s.found_key, s.found_own};
    __syncthreads();
    return p;
}

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

template <int TYPE> __global__ __launch_bounds__(1024) void sample_kernel(SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Shared &s = *reinterpret_cast<Shared *>(lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const size_t r = blockIdx.x;
    const Row<TYPE> row{static_cast<const real_t<TYPE> *>(a.logits) + r * (size_t)a.stride, a.vocab};
    for (int i = tid; i < BINS; i += blockDim.x) {
        s.count[0][i] = 0;
        s.mass[0][i] = 0;
    }
    for (int i = tid; i < 256; i += blockDim.x) s.table[i] = exp2(i * (-1.0 / PER_OCTAVE));
    float top = -__builtin_inff();
    bool bad = false;
    for (int c = 8 * tid; c < a.vocab; c += 8 * blockDim.x) {
        Real8<TYPE> v;
        v.load(row.l + c, a.vocab - c, -__builtin_inff());
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top = fmaxf(top, v[j]);
            bad |= !(v[j] < __builtin_inff());
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const bool any_bad = __any(bad);
    if (lane == 0) {
        s.wave_top[wave] = top;
        s.wave_bad[wave] = any_bad;
    }
    const float T = a.temperature ? a.temperature[r] : 1.0f, top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f, u = a.uniform[r];
    const int top_k = a.top_k ? a.top_k[r] : 0;
    __syncthreads();
    bad = !(T >= 0.0f) || top_p != top_p || min_p != min_p || u != u;
    for (int i = 0; i < waves; ++i) {
        top = fmaxf(top, s.wave_top[i]);
        bad |= s.wave_bad[i] != 0;
    }
    if (bad || top == -__builtin_inff()) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = bad ? __builtin_nanf("") : -__builtin_inff();
            if (a.kept) a.kept[r] = 0;
        }
        return;
    }
    const bool first_only = T == 0.0f || top_k == 1;
    const Weigh w{(double)top, PER_OCTAVE * 0x1.71547652b82fep+0 / (T == 0.0f ? 1.0 : (double)T), a.bits, s.table};         // log2 e
    const double least = fmin((double)min_p, 1.0);
    uint64_t mass_min = 0, count_min = 0;
    row.each([&](float l, int) {
        const double t = w.distance(l), e = w.weight(t, w.bits);
        const uint64_t m = Weigh::rounded(e);
        atomicAdd(&s.count[0][Weigh::bin(t)], 1u);
        atomicAdd((unsigned long long *)&s.mass[0][Weigh::bin(t)], (unsigned long long)m);
        if (e >= __builtin_ldexp(least, w.bits)) {
            mass_min += m;
            ++count_min;
        }
    });
    __syncthreads();
    uint64_t count, mass, m = 0, c = 0, all;
    for (int i = tid; i < BINS; i += blockDim.x) {
        c += s.count[0][i];
        m += s.mass[0][i];
    }
    scan(c, s.wave_count, count);
    scan(m, s.wave_mass, mass);
    scan(count_min, s.wave_count, all);
    count_min = all;
    scan(mass_min, s.wave_mass, all);
    mass_min = all;
    if (first_only) {
        count = 1;
        mass = 1ull << a.bits;
    } else {
        if (top_k > 0 && (uint64_t)top_k < count) {
            const Place p = search(s, row, w, false, (uint64_t)top_k);
            count = p.count;
            mass = p.mass;
        }
        if (top_p < 1.0f) {
            uint64_t target = top_p > 0.0f ? share(top_p, mass, true) : 1;
            const Place p = search(s, row, w, true, target ? target : 1);
            count = p.count;
            mass = p.mass;
        }
        if (min_p > 0.0f && count_min < count) {
            count = count_min;
            mass = mass_min;
        }
    }
    const float clamped = u < 0.0f ? 0.0f : u < 1.0f ? u : 0x1.fffffep-1f;
    const Place p = search(s, row, w, true, share(clamped, mass, false) + 1);
    if (tid == 0) {
        const int token = (int)(uint32_t)p.key;
        a.token[r] = token;
        if (a.kept) a.kept[r] = (int)count;
        if (a.logprob) {
            // (l - top) / T - log(sum): the token's weight as it is, not as it was rounded
            const double d = T == 0.0f ? 0.0 : ((double)(float)row.l[token] - (double)top) / (double)T;
            a.logprob[r] = first_only ? 0.0f : fminf((float)(d - log(__builtin_ldexp((double)mass, -a.bits))), 0.0f);
        }
    }
}

}  // namespace

size_t sample_workspace_bytes(int, int) { return 0; }
bool sample_needs(int, int) { return false; }

xnor_status launch_sample(const void *logits, long long stride, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                          const float *uniform, int32_t *token, float *logprob, int32_t *kept, void *, int rows, int vocab, int type, hipStream_t stream)
{
    int b = 0;
    while ((1ll << b) < vocab) ++b;
    const SampleArgs a{logits, temperature, top_p, min_p, uniform, top_k, token, kept, logprob, stride, rows, vocab, b > 18 ? 62 - b : 44};
    const int threads = vocab > 8192 ? 1024 : vocab > 2048 ? 512 : 256;
    xnor_status status = XNOR_OK;
    by_type(type, [&](auto t) {
        auto kernel = sample_kernel<t()>;
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shared)) != hipSuccess) {
            status = XNOR_ERR_HIP;
            return;
        }
        kernel<<<dim3((unsigned)rows), dim3((unsigned)threads), sizeof(Shared), stream>>>(a);
        status = hip_status(hipGetLastError());
    });
    return status;
}

}  // namespace xnor
