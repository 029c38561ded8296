// Products of many rows with 4-bit weights: rows staged once as operands, then tiles of 256 outputs x 128 rows or 64 x 64.
#include "xnor_internal.h"
#include "lowbit.h"
#include "w4_form.h"
#include "w4_image.h"
#include <algorithm>
#include <cmath>

namespace xnor {

namespace {

static_assert(ROWS_I8 == W4_8_BITS);

constexpr int TILE = 16, BLOCK = 8;         // rows or outputs of a matrix instruction, such tiles of a workgroup's side

// What the rows become (the first kernel writes it, the second reads it), in a workspace of the caller's:
//   operands  [block of 128 rows][chunk of 128 inputs][part][tile of 16 rows][step][lane][16 bytes]: 16 bits, 4 steps of 32 inputs; 8 bits, 2 steps
//             of 64.  Tiles past the last row are not written: they meet no result that is kept
//   sums      [tile of 16 rows][quad of groups][lane] float32, 16 bits only: the groups' sums of SHARE x, lane 16 i + r is row r, group i of the quad
//   scales    [tile of 16 rows][group][row] float32, 8-bit rows with scales of groups only
struct Staged {
    int blocks, chunks, parts, groups, quads;
    bool bytes;
    __host__ __device__ Staged(int rows, int in, int group, int form)
        : blocks((rows + TILE * BLOCK - 1) / (TILE * BLOCK)), chunks((in + 127) / 128), parts(form == ROWS_F32 ? 3 : 1),
          groups((in + group - 1) / group), quads(form == ROWS_I8 ? 0 : (groups + 3) / 4), bytes(form == ROWS_I8) {}
    __host__ __device__ int tile_bytes() const { return bytes ? 2048 : 4096; }
    __host__ __device__ size_t sums_at() const { return (size_t)blocks * chunks * parts * BLOCK * tile_bytes(); }
    __host__ __device__ size_t scales_at() const { return sums_at() + (size_t)blocks * BLOCK * quads * 256; }
    __host__ __device__ size_t total() const { return scales_at() + (bytes ? (size_t)blocks * BLOCK * groups * 64 : 0); }
};

// The factors of what is taken out, BACK between them: a group's sum and 32 scales stay within float32's range.
template <int X> constexpr float SHARE = Form<X>::BACK == 1.0f ? 1.0f : 1.0f / 128.0f;

// What four groups' offset and zero points add to the totals of 16 outputs x 16 rows, taken out: - scale (OFFSET + zero) of a lane's output and group (its
// quarter) times the group's sum of a lane's row, four groups in one instruction.  It multiplies and adds in 32 bits: bfloat16 parts of both factors in the
// instructions of the products leave a part of every sum out that has a sign (2.9e-6 of the results' size where this leaves 5e-7).
template <int X> __device__ __forceinline__ f32x4 less_offset(f32x4 total, float scale, uint8_t zero, float sum)
{
    constexpr float rest = 1.0f / (Form<X>::BACK * SHARE<X>);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(-(scale * __builtin_fmaf((float)zero, rest, Form<X>::OFFSET * rest)), sum, total, 0, 0, 0);
}

struct StageArgs {
    const void *x;
    const float *x_scale;
    uint8_t *staged;
    long long x_stride;
    int rows, in, group, x_group, x_groups;
};

// A wave stages 16 rows x 128 inputs.  What bounds it: memory (2048 x 4096 bfloat16 7.4 us, 34 MB, 4.6 TB/s), for few rows the launch (256 x 9216 8 bits
// 4 us).
template <int X>
__global__ __launch_bounds__(256) void w4_stage_kernel(StageArgs a)
{
    typedef Form<X> F;
    const Staged st(a.rows, a.in, a.group, X);
    const int lane = threadIdx.x & 63, r = lane & 15, quarter = lane >> 4;
    const int chunk = blockIdx.y * 4 + (threadIdx.x >> 6), tile = blockIdx.x;
    if (chunk >= st.chunks) return;
    const int row = tile * TILE + r;
    const bool real = row < a.rows;
    constexpr int XBYTES = X == ROWS_F32 ? 4 : X == ROWS_I8 ? 1 : 2;
    const char *x = static_cast<const char *>(a.x) + (size_t)(real ? row : 0) * a.x_stride * XBYTES;
    u32x4 *out = reinterpret_cast<u32x4 *>(a.staged) +
                 (((size_t)(tile / BLOCK) * st.chunks + chunk) * st.parts * BLOCK + tile % BLOCK) * (st.tile_bytes() / 16) + lane;
    Eight<X> v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int k = 128 * chunk + 32 * j + 8 * quarter;
        v[j].load(x, k, real ? a.in - k : 0);
    }
    const int steps = a.group / 32, per_chunk = 4 / steps, first = chunk * per_chunk;
    if constexpr (X == ROWS_I8) {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            long b[2];
            v[j].operands(b);
            v[j + 1].operands(b + 1);
            out[(j / 2) * 64] = u32x4{(uint32_t)b[0], (uint32_t)(b[0] >> 32), (uint32_t)b[1], (uint32_t)(b[1] >> 32)};
        }
        if (!a.x_group) return;
        const int g = first + quarter;
        if (quarter < per_chunk && g < st.groups)
            reinterpret_cast<float *>(a.staged + st.scales_at())[((size_t)tile * st.groups + g) * 16 + r] =
                real ? a.x_scale[(size_t)row * a.x_groups + (int)((long long)g * a.group / a.x_group)] : 0.0f;
    } else {
        float sum[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            typename F::operand_t b[F::PARTS];
            v[j].operands(b);
#pragma unroll
            for (int p = 0; p < F::PARTS; ++p) out[(size_t)p * BLOCK * 256 + j * 64] = b[p];
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v[j].v[i], SHARE<X>, s);
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            sum[j] = s;
        }
        // the groups' sums, and zeros up to a whole quad behind the last
        if (steps >= 2) {
            sum[0] += sum[1];
            sum[1] = sum[2] + sum[3];
        }
        if (steps == 4) sum[0] += sum[1];
        float *sums = reinterpret_cast<float *>(a.staged + st.sums_at()) + (size_t)tile * st.quads * 64;
        const int last = chunk == st.chunks - 1 ? 4 * st.quads : first + per_chunk;
        for (int g = first + quarter; g < last; g += 4) {
            const int i = g - first;
            sums[(size_t)g * 16 + r] = i >= per_chunk ? 0.0f : i == 0 ? sum[0] : i == 1 ? sum[1] : i == 2 ? sum[2] : sum[3];
        }
    }
}

struct TileArgs {
    const uint8_t *staged, *image;
    const float *x_scale;
    void *y;
    int rows, in, out, type, form;
    int row_blocks, out_blocks;
};

// The lane's number, made anew: what a loop without a register to spare does not keep (a spilled one would come back behind all loads on their way).
__device__ __forceinline__ int lane_anew()
{
    uint32_t none = 0;
    asm volatile("" : "+s"(none));
    return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(1))) uint8_t global_u8;

__device__ __forceinline__ void to_lds(const uint8_t *from, uint8_t *to)        // 16 bytes per lane, to + 16 * lane
{
    __builtin_amdgcn_global_load_lds((global_u8 *)from, (lds_u8 *)to, 16, 0, 0);
}

// STEPS of 32 inputs per group.  2 * SIDE waves, each 64 outputs x 64 rows, together 64 * SIDE outputs x 128 rows.  All a chunk needs (the rows' operands,
// codes, scales, zero points) goes straight to one of BUFFERS places in LDS, BUFFERS - 1 chunks ahead, one barrier per chunk.  Every wave issues
// the same number of loads for a chunk, so that it can wait for its oldest chunk alone.  GROUPED: 8-bit rows with scales of groups.
// What bounds it: matrix and vector instructions, of which the waves leave a chunk's barrier with the same ones to do, so that they hardly overlap.  2048 bfloat16
// rows 4096 -> 8192, groups of 128: 141 us with the staging, 0.98 PFLOP/s (a library's product with bfloat16 weights 99); of the cycles, at 2.2 GHz, the matrix
// pipes are busy in 0.44 and vector instructions take 0.35.  Groups of 64 199 us, of 32 219 (four times the scaling; what is taken out is half as much matrix
// work again).  8 bits 120, 208, 316: 0.23 and 0.61 in groups of 128 (converting, scaling twice, widening).  Float32 rows, three products: 360, 497, 505.
// Tried when groups of 128 took 138: instructions of 32 x 32 results 156, the next chunk's first operands read ahead of the barrier 149.
template <int X, int STEPS, bool GROUPED, int SIDE> struct TilePlace {
    static constexpr int WAVES = 2 * SIDE, PER_CHUNK = 4 / STEPS, TB = X == ROWS_I8 ? 2048 : 4096;
    static constexpr int ROWS = 0, CODES = BLOCK * TB, SCALES = CODES + SIDE * 4096, FACTORS = 4 * PER_CHUNK * 64;      // of four tiles
    static constexpr int ROW_SCALES = SCALES + SIDE * FACTORS, ZEROS = ROW_SCALES + (GROUPED ? 2 * FACTORS : 0);
    static constexpr int BYTES = ZEROS + (X == ROWS_I8 ? SIDE * FACTORS / 4 : 0);
    static constexpr int LOADS = BLOCK * TB / (WAVES * 1024) + 2 + 1 + (GROUPED ? 1 : 0) + (X == ROWS_I8 ? 1 : 0);
};

template <int X, int STEPS, bool GROUPED, int SIDE, int BUFFERS>
__global__ __launch_bounds__(128 * SIDE) void w4_tiles_kernel(TileArgs a)
{
    typedef Form<X> F;
    typedef TilePlace<X, STEPS, GROUPED, SIDE> P;
    constexpr int WAVES = P::WAVES, AHEAD = BUFFERS - 1, TB = P::TB, PER_CHUNK = P::PER_CHUNK;
    // 16 bits: groups of 32 leave no register for a lane's places; groups of 128 leave enough for what is taken out to be loaded ahead of a step's products
    // (behind them 144 us in place of 140)
    constexpr bool SPARE = X == ROWS_I8 || STEPS > 1, EARLY = STEPS == 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const W4Layout l(a.out, a.in, 32 * STEPS);
    const Staged st(a.rows, a.in, 32 * STEPS, a.form);
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wo = wave % SIDE, wr = wave / SIDE;
    // workgroups go to the XCDs in turn: each takes a run of neighbouring tiles
    const int count = a.row_blocks * a.out_blocks, per_xcd = (count + 7) / 8;
    const int id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || id >= count) return;
    // (in strips of four blocks of rows: the workgroups of an XCD read 4 blocks of rows and 8 of codes at a time, 256 KB per chunk; whole columns of blocks
    // 544 KB.  8192 bfloat16 rows 4096 -> 8192 556 us, by columns 587)
    constexpr int STRIP = 4;
    const int strip = id / (STRIP * a.out_blocks), within = id - strip * STRIP * a.out_blocks, high = min(STRIP, a.row_blocks - strip * STRIP);
    const int ob = within / high, rb = strip * STRIP + within - ob * high;
    const int otile = ob * 4 * SIDE + wo * 4, rtile = rb * BLOCK + wr * 4;
    const int parts = st.parts, steps = st.chunks * parts;

    // (tiles past the last are the last once more)
    const uint8_t *scales = a.image + l.scale_at(), *zeros = a.image + l.zero_at();
    const uint8_t *rows_from = a.staged + (size_t)rb * steps * BLOCK * TB;
    const uint8_t *codes_from[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) codes_from[i] = a.image + (size_t)min(ob * 4 * SIDE + wave * 2 + i, l.tiles - 1) * l.chunks * 1024;
    // scales and zero points of a wave's four tiles: it loads a half of them, the wave of the other rows the other; the rows' scales: a share of each
    // wave with the same rows.  Lanes: tile, group of the chunk, quarter of 16 factors (a lane per 16 bytes)
    constexpr int SCALE_LANES = P::FACTORS / 32, ROW_LANES = P::FACTORS / 16 / SIDE, ZERO_LANES = P::FACTORS / 128;
    const int otile0 = min(otile, l.tiles - 1), more = l.tiles - 1 - otile0;
    const int f = min(lane, SCALE_LANES - 1) + wr * SCALE_LANES, fr = min(lane, ROW_LANES - 1) + wo * ROW_LANES, fz = min(lane, ZERO_LANES - 1) + wr * ZERO_LANES;
    const uint8_t *scales_from = scales + (size_t)otile0 * l.groups * 64, *zeros_from = zeros + (size_t)otile0 * l.groups * 16;
    const uint8_t *row_scales_from = a.staged + st.scales_at() + (size_t)rtile * l.groups * 64;
    const uint32_t scale_off = (uint32_t)min(f / (4 * PER_CHUNK), more) * l.groups * 64 + (f & 3) * 16;
    const uint32_t row_off = (uint32_t)(fr / (4 * PER_CHUNK)) * l.groups * 64 + (fr & 3) * 16;
    const uint32_t zero_off = (uint32_t)min(fz / PER_CHUNK, more) * l.groups * 16;
    const uint32_t at = tid * 16, lane_at = lane * 16;
    // step = chunk * parts + part; a group past the last meets sums of zero
    auto fetch = [&](int step, int place) {
        const int c = parts == 1 ? step : (int)(__umulhi((uint32_t)step, 0xaaaaaaabu) >> 1), g0 = c * PER_CHUNK;
        uint8_t *to = lds + place * P::BYTES;
        const uint8_t *from = rows_from + (size_t)step * BLOCK * TB;
#pragma unroll
        for (int i = 0; i < BLOCK * TB / (WAVES * 1024); ++i) to_lds(from + i * WAVES * 1024 + at, to + (i * WAVES + wave) * 1024);
#pragma unroll
        for (int i = 0; i < 2; ++i) to_lds(codes_from[i] + (size_t)c * 1024 + lane_at, to + P::CODES + (wave * 2 + i) * 1024);
        if constexpr (SPARE) {
            if (lane < SCALE_LANES)
                to_lds(scales_from + (scale_off + (uint32_t)min(g0 + f / 4 % PER_CHUNK, l.groups - 1) * 64), to + P::SCALES + wo * P::FACTORS + wr * SCALE_LANES * 16);
        } else if (const int now = lane_anew(); now < SCALE_LANES) {
            const int f = now + wr * SCALE_LANES;
            to_lds(scales_from + ((uint32_t)min(f / (4 * PER_CHUNK), more) * l.groups + min(g0 + f / 4 % PER_CHUNK, l.groups - 1)) * 64 + (f & 3) * 16,
                   to + P::SCALES + wo * P::FACTORS + wr * SCALE_LANES * 16);
        }
        if (GROUPED && lane < ROW_LANES)
            to_lds(row_scales_from + (row_off + (uint32_t)min(g0 + fr / 4 % PER_CHUNK, l.groups - 1) * 64),
                   to + P::ROW_SCALES + wr * P::FACTORS + wo * ROW_LANES * 16);
        if (X == ROWS_I8 && lane < ZERO_LANES)
            to_lds(zeros_from + (zero_off + (uint32_t)min(g0 + fz % PER_CHUNK, l.groups - 1) * 16), to + P::ZEROS + wo * P::FACTORS / 4 + wr * ZERO_LANES * 16);
    };
    f32x4 total[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) total[i][j] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) fetch(min(r, steps - 1), r);
    // What the offset and the zero points add is taken out beside the sums that hold it, in the middle of every four groups, so that the total is never
    // further from the result than their terms.  2048 float32 rows of one sign, 9216 -> 4096: off by 5.6e-7 of the results' size in groups of 128, 7.9e-7 of
    // 32 (a 32-bit library product of the real weights 3.9e-7; all groups taken out at once 1.1e-5 and 6.4e-5).
    const int per_quad = STEPS * parts;          // steps of four groups
    int quad = 0, due = X == ROWS_I8 ? -1 : min((per_quad - 1) / 2, steps - 1);
    float sum_out[4], scale_out[4];
    uint32_t zeros_out[4];
    auto load_out = [&]() {
        const int now = SPARE ? lane : lane_anew();
        const float *sums = reinterpret_cast<const float *>(a.staged + st.sums_at()) + ((size_t)rtile * st.quads + quad) * 64;
        const uint32_t at = min(4 * quad + (now >> 4), l.groups - 1) * 16 + (now & 15);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t tile = (size_t)min(otile + i, l.tiles - 1) * l.groups * 16;
            sum_out[i] = (sums + (size_t)i * st.quads * 64)[now];
            scale_out[i] = (reinterpret_cast<const float *>(scales) + tile)[at];
            zeros_out[i] = (zeros + tile)[at];
        }
    };
    auto take_out = [&]() {
        if constexpr (X != ROWS_I8)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) total[i][j] = less_offset<X>(total[i][j], scale_out[i], (uint8_t)zeros_out[i], sum_out[j]);
        ++quad;
        due = quad < st.quads ? min(due + per_quad, steps - 1) : -1;
    };
    // A group's sums wait in acc, with the factors they are scaled by, until the first product of the next group takes their place: the scaling
    // fills the time that the next chunk's operands take from LDS, and that a product takes.
    constexpr int WIDE = X == ROWS_I8 && STEPS >= 2 ? 2 : 1, PHASES = 4 / WIDE;        // steps of 32 inputs per product, products per chunk
    typename F::acc_t acc[4][4];
    f32x4 factor[4];
    float row_factor[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        factor[i] = f32x4{0, 0, 0, 0};
        row_factor[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = typename F::acc_t{0, 0, 0, 0};
    }
    auto rescale = [&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float part = (float)acc[i][j][v];
                if (GROUPED) part *= row_factor[j];
                total[i][j][v] = __builtin_fmaf(factor[i][v], part, total[i][j][v]);
            }
    };
    int place = 0;
    for (int s = 0; s < steps; ++s) {
        // this chunk's loads are over (LOADS of each later one may not be), everybody's; and nobody reads the place of the chunk before
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * P::LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (X != ROWS_I8 && EARLY && s == due) load_out();
        const uint8_t *here = lds + place * P::BYTES, *x = here + wr * 4 * TB + lane_at, *wc = here + P::CODES + wo * 4096 + lane_at;
        const uint8_t *sw = here + P::SCALES + wo * P::FACTORS + quarter * 16, *sx = here + P::ROW_SCALES + wr * P::FACTORS + col * 4;
        const uint8_t *zero = here + P::ZEROS + wo * P::FACTORS / 4 + col;
        u32x4 w[4], b[2][4];
        uint32_t z[4];
        auto read_rows = [&](int phase) {           // (8 bits: one load holds 64 inputs)
            const int t = X == ROWS_I8 ? phase * WIDE / 2 : phase;
            if (X == ROWS_I8 && WIDE == 1 && phase % 2) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) b[t & 1][j] = *reinterpret_cast<const u32x4 *>(x + j * TB + t * 1024);
        };
        read_rows(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const u32x4 *>(wc + i * 1024);
        fetch(min(s + AHEAD, steps - 1), place == 0 ? BUFFERS - 1 : place - 1);          // (past the end: the last chunk once more, which nobody reads)
        place = place == BUFFERS - 1 ? 0 : place + 1;
#pragma unroll
        for (int phase = 0; phase < PHASES; ++phase) {
            const bool starts = phase * WIDE % STEPS == 0;
            const int g = phase * WIDE / STEPS, t = X == ROWS_I8 ? phase * WIDE / 2 : phase;
            if (X == ROWS_I8 && starts)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = zero[(i * PER_CHUNK + g) * 16] * 0x01010101u;
            if (phase + 1 < PHASES) read_rows(phase + 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (starts) {
                    rescale(i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = typename F::acc_t{0, 0, 0, 0};
                }
                if constexpr (X != ROWS_I8) {
                    const auto wide = F::widen(w[i][phase]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = F::mfma(wide, b[t & 1][j], acc[i][j]);
                } else if constexpr (STEPS == 1) {          // (two groups in the 64 inputs of a load)
                    const long wide = F::widen(w[i][phase], z[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = F::mfma(wide, (long)((uint64_t)b[t & 1][j][2 * (phase & 1)] | (uint64_t)b[t & 1][j][2 * (phase & 1) + 1] << 32), acc[i][j]);
                } else {
                    const uint32_t c0 = w[i][2 * phase], c1 = w[i][2 * phase + 1];
                    const i32x4 wide{(int)F::minus(c0, z[i]), (int)F::minus(c0 >> 4, z[i]), (int)F::minus(c1, z[i]), (int)F::minus(c1 >> 4, z[i])};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wide, __builtin_bit_cast(i32x4, b[t & 1][j]), acc[i][j], 0, 0, 0);
                }
            }
            if (starts) {
#pragma unroll
                for (int i = 0; i < 4; ++i) factor[i] = *reinterpret_cast<const f32x4 *>(sw + (i * PER_CHUNK + g) * 64);
                if (GROUPED)
#pragma unroll
                    for (int j = 0; j < 4; ++j) row_factor[j] = *reinterpret_cast<const float *>(sx + (j * PER_CHUNK + g) * 64);
            }
        }
        if (X != ROWS_I8 && s == due) {
            if (!EARLY) load_out();
            take_out();
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);                           // lgkmcnt(0): its reads of the place are over at the next barrier
        asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) rescale(i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = (rtile + j) * TILE + col;
        if (row >= a.rows) continue;
        const float c = X == ROWS_I8 && !GROUPED ? a.x_scale[row] : 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int o = (otile + i) * TILE + 4 * quarter;
            f32x4 v = total[i][j];
            if constexpr (X != ROWS_I8) v *= F::BACK;
            else if (!GROUPED) v *= c;
            store_four(a.y, a.type, (size_t)row * a.out + o, v, a.out - o);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                     // (the loads past the end are into this workgroup's LDS)
}

// The same sums where there are too few tiles of that size: a workgroup makes 64 outputs x 64 rows, its eight waves take every eighth chunk (its parts
// one after another), operands straight to registers, and add their sums in LDS.
// What bounds it: the caches, and vector instructions between a step's loads (256 bfloat16 rows 9216 -> 4096: each workgroup reads 1.5 MB, some 60 bytes per ns and
// CU; 30 us with the staging.  8 bits 25, vector instructions half of the cycles).  The same loads a chunk ahead, through LDS, were 1 to 2 us slower.
template <int X, int STEPS, bool GROUPED>
__global__ __launch_bounds__(512) void w4_waves_kernel(TileArgs a)
{
    typedef Form<X> F;
    constexpr int WAVES = 8, TB = X == ROWS_I8 ? 2048 : 4096, PER_CHUNK = 4 / STEPS, PITCH = 68;
    extern __shared__ __attribute__((aligned(16))) float red[];             // [WAVES][64 rows][PITCH]
    const W4Layout l(a.out, a.in, 32 * STEPS);
    const Staged st(a.rows, a.in, 32 * STEPS, a.form);
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int otile = blockIdx.x * 4, rtile = blockIdx.y * 4;
    const u32x4 *codes[4];
    const float *scales[4];
    const uint8_t *zeros[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const size_t tile = min(otile + i, l.tiles - 1);
        codes[i] = reinterpret_cast<const u32x4 *>(a.image) + tile * l.chunks * 64 + lane;
        scales[i] = reinterpret_cast<const float *>(a.image + l.scale_at()) + tile * l.groups * 16;
        zeros[i] = a.image + l.zero_at() + tile * l.groups * 16 + col;
    }
    const float *row_scales = reinterpret_cast<const float *>(a.staged + st.scales_at()) + (size_t)rtile * l.groups * 16 + col;
    const float *sums = reinterpret_cast<const float *>(a.staged + st.sums_at()) + (size_t)rtile * st.quads * 64;
    const u32x4 *rows_from = reinterpret_cast<const u32x4 *>(a.staged + ((size_t)(rtile / BLOCK) * st.chunks * st.parts * BLOCK + rtile % BLOCK) * TB) + lane;
    f32x4 total[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) total[i][j] = f32x4{0, 0, 0, 0};
    constexpr int READS = TB / 1024;
    const int steps = st.chunks * st.parts;
    for (int s = wave; s < steps; s += WAVES) {
        const int chunk = st.parts == 1 ? s : (int)(__umulhi((uint32_t)s, 0xaaaaaaabu) >> 1);
        // (all loads of a step at once: their trips are what a step takes)
        u32x4 w[4], b[READS][4];
        f32x4 f[PER_CHUNK][4];
        float c[PER_CHUNK][4];
        uint32_t z[PER_CHUNK][4];
        // What the offset and the zero points add to the wave's next STEPS chunks, four groups, is taken out before their sums (as in w4_tiles_kernel; 256
        // float32 rows of one sign, 9216 -> 4096: off by 3e-7 to 6.5e-7).  The lane's group of them:
        const int own = min((chunk + quarter / PER_CHUNK * WAVES) * PER_CHUNK + quarter % PER_CHUNK, l.groups) * 16 + col;
        const bool real = own < l.groups * 16;
        const int own_at = real ? own : col;
        float sum[4], scale[4];
        uint8_t zero_point[4];
        if (X != ROWS_I8)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[i] = sums[(size_t)i * st.quads * 64 + own_at];
                scale[i] = scales[i][own_at];
                zero_point[i] = zeros[i][own_at - col];
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = codes[i][(size_t)chunk * 64];
#pragma unroll
        for (int t = 0; t < READS; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) b[t][j] = rows_from[(size_t)s * (BLOCK * TB / 16) + j * (TB / 16) + t * 64];
#pragma unroll
        for (int n = 0; n < PER_CHUNK; ++n) {
            const size_t g = min(chunk * PER_CHUNK + n, l.groups - 1) * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[n][i] = *reinterpret_cast<const f32x4 *>(scales[i] + g + 4 * quarter);
                if (X == ROWS_I8) z[n][i] = zeros[i][g];
                if (GROUPED) c[n][i] = row_scales[(size_t)i * l.groups * 16 + g];
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (X != ROWS_I8)
            if (s == chunk * st.parts && chunk / WAVES % STEPS == 0)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) total[i][j] = less_offset<X>(total[i][j], real ? scale[i] : 0.0f, zero_point[i], sum[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typename F::acc_t acc[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t zero = X == ROWS_I8 ? z[t / STEPS][i] * 0x01010101u : 0;
                if (t % STEPS == 0)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = typename F::acc_t{0, 0, 0, 0};
                if constexpr (X != ROWS_I8) {
                    const auto wide = F::widen(w[i][t]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = F::mfma(wide, b[t][j], acc[j]);
                } else if constexpr (STEPS == 1) {          // (two groups in the 64 inputs of a load)
                    const long wide = F::widen(w[i][t], zero);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[j] = F::mfma(wide, (long)((uint64_t)b[t / 2][j][2 * (t & 1)] | (uint64_t)b[t / 2][j][2 * (t & 1) + 1] << 32), acc[j]);
                } else if (t % 2 == 0) {
                    const i32x4 wide{(int)F::minus(w[i][t], zero), (int)F::minus(w[i][t] >> 4, zero), (int)F::minus(w[i][t + 1], zero),
                                     (int)F::minus(w[i][t + 1] >> 4, zero)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wide, __builtin_bit_cast(i32x4, b[t / 2][j]), acc[j], 0, 0, 0);
                }
                if (t % STEPS != STEPS - 1) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float part = (float)acc[j][v];
                        if (GROUPED) part *= c[t / STEPS][j];
                        total[i][j][v] = __builtin_fmaf(f[t / STEPS][i][v], part, total[i][j][v]);
                    }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4 *>(red + (wave * 64 + 16 * j + col) * PITCH + 16 * i + 4 * quarter) = total[i][j];
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int r = (tid >> 4) + 32 * p, q = (tid & 15) * 4, row = rtile * TILE + r, o = otile * TILE + q;
        if (row >= a.rows) continue;
        f32x4 v = *reinterpret_cast<const f32x4 *>(red + r * PITCH + q);
#pragma unroll
        for (int k = 1; k < WAVES; ++k) v += *reinterpret_cast<const f32x4 *>(red + (k * 64 + r) * PITCH + q);
        if constexpr (X != ROWS_I8) v *= F::BACK;
        else if (!GROUPED) v *= a.x_scale[row];
        store_four(a.y, a.type, (size_t)row * a.out + o, v, a.out - o);
    }
}

constexpr int SIDE = 4;             // waves of w4_tiles_kernel along the outputs, 64 of them each

template <int X, bool GROUPED> xnor_status launch_waves(const TileArgs &a, int group, hipStream_t stream)
{
    constexpr unsigned lds = 8 * 64 * 68 * sizeof(float);
    const dim3 grid((unsigned)((a.out + 63) / 64), (unsigned)((a.rows + 63) / 64));
    auto go = [&](auto kernel) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return XNOR_ERR_HIP;
        kernel<<<grid, dim3(512), lds, stream>>>(a);
        return hip_status(hipGetLastError());
    };
    if (group == 32) return go(w4_waves_kernel<X, 1, GROUPED>);
    if (group == 64) return go(w4_waves_kernel<X, 2, GROUPED>);
    return go(w4_waves_kernel<X, 4, GROUPED>);
}

template <int X, bool GROUPED> xnor_status launch_tiles(const TileArgs &a, int group, hipStream_t stream)
{
    constexpr int BUFFERS = X == ROWS_I8 ? 4 : 3;
    const long long count = (long long)a.row_blocks * a.out_blocks;
    if (count > 0xffffff00LL / (128 * SIDE)) return XNOR_ERR_SHAPE;
    const dim3 grid((unsigned)((count + 7) / 8 * 8));
    auto go = [&](auto kernel, unsigned lds) {
        if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
            return XNOR_ERR_HIP;
        kernel<<<grid, dim3(128 * SIDE), lds, stream>>>(a);
        return hip_status(hipGetLastError());
    };
    if (group == 32) return go(w4_tiles_kernel<X, 1, GROUPED, SIDE, BUFFERS>, BUFFERS * TilePlace<X, 1, GROUPED, SIDE>::BYTES);
    if (group == 64) return go(w4_tiles_kernel<X, 2, GROUPED, SIDE, BUFFERS>, BUFFERS * TilePlace<X, 2, GROUPED, SIDE>::BYTES);
    return go(w4_tiles_kernel<X, 4, GROUPED, SIDE, BUFFERS>, BUFFERS * TilePlace<X, 4, GROUPED, SIDE>::BYTES);
}

}  // namespace

// Rounds of a workgroup per CU.
static double rounds(int out, int outs, int rows, int height)
{
    return std::ceil((double)((out + outs - 1) / outs) * ((rows + height - 1) / height) / 256);
}

// Which kernel takes a product: the shortest of their times in us, fitted to 175 products (inputs 256 to 9216, outputs 256 to 32000, 1 to 2048 rows, every type and
// group, half of them no multiple of anything), of which it picks one that is more than a tenth slower than the best once.
// w4_rows_kernel reads all rows' inputs in every workgroup, slower where they start at odd addresses, but is one launch; the others stage the rows first.
// More tiles per workgroup read the inputs less often, and leave fewer workgroups: one, two and four tiles, one bfloat16 row 9216 -> 4096 6.5, 9.1, 14.7; 32
// rows 20, 13.6, 16.8; 64 rows 38, 25, 17; 8 8-bit rows 4096 -> 32000 24, 16, 14.7; 128 float32 rows 1003 -> 1000 6.4, 5.0, 6.4.
// Tiles of 64 x 64 whose inputs eight waves share fill the chip where few of 256 x 128 would not.  By rows, by waves, by tiles: 64 bfloat16 rows 9216 -> 4096
// 17, 26, 138; 48 rows 4096 -> 16384 21, 18, 65; 128 rows 4096 -> 8192 34, 19, 75, 4097 -> 8192 70, 20, 77; 247 8-bit rows 8538 -> 31744 in groups of 32 737, 258,
// 316; 2048 bfloat16 rows 4096 -> 8192 -, 189, 141.
static W4Choice by_rows(int rows, int in, int out, int form)
{
    const bool f32 = form == ROWS_F32, i8 = form == ROWS_I8;
    const double by_eight = 8 * std::ceil((in + 127) / 128 / 8.0);          // (eight waves share the chunks)
    const double operand = f32 ? 2.1 : i8 ? (in % 4 ? 1.5 : 1.3) : in % 2 ? 2.2 : 1.0;
    W4Choice best{W4_ROWS, 0, 0.0};
    for (int tiles : {1, 2, 4}) {
        const double chunk = tiles == 1 ? 0.1 : tiles == 2 ? 0.145 : 0.185;
        const double time = 2.6 + rounds(out, 16 * tiles, rows, 16) * (0.6 + chunk * operand * by_eight);
        if (best.tiles == 0 || time < best.time) best = {W4_ROWS, tiles, time};
    }
    if (rows > 16 * 65535) best.time = HUGE_VAL;                            // (a launch's second dimension)
    return best;
}
static W4Choice staged(int rows, int in, int out, int group, int form)
{
    const bool i8 = form == ROWS_I8;
    const double steps = (in + 127) / 128 * (form == ROWS_F32 ? 3.0 : 1.0);
    // a group's scaling weighs more where groups are short
    const double scaled = group == 32 ? 1.4 : group == 64 ? 1.08 : 1.0, tile_scaled = group == 32 ? (i8 ? 2.3 : 1.45) : group == 64 ? (i8 ? 1.1 : 1.35) : 1.0;
    const double by_waves = 3.5 + rounds(out, 64, rows, 64) * (2.2 + scaled * (i8 ? 1.6 : 2.5) * std::ceil(steps / 8));
    const double by_tiles = 10 + tile_scaled * (i8 ? 1.6 : 2.3) * steps * rounds(out, 64 * SIDE, rows, TILE * BLOCK);
    return by_tiles < by_waves ? W4Choice{W4_TILES, 0, by_tiles} : W4Choice{W4_WAVES, 0, by_waves};
}
W4Choice w4_choice(int rows, int in, int out, int group, int form)
{
    const W4Choice one = by_rows(rows, in, out, form), two = staged(rows, in, out, group, form);
    return two.time < one.time ? two : one;
}

bool w4_linear_needs(int rows, int in, int out, int group, int form) { return w4_choice(rows, in, out, group, form).kernel != W4_ROWS; }

// Enough for up to `rows` rows of any type.  Neither time falls as rows grows, so rows are staged nowhere up to where w4_rows_kernel takes no longer than the
// others for one row.
size_t w4_linear_workspace_bytes(int rows, int in, int out, int group)
{
    size_t most = 0;
    for (int form : {(int)ROWS_F32, (int)ROWS_BF16, (int)ROWS_I8})
        if (by_rows(rows, in, out, form).time > staged(1, in, out, group, form).time) most = std::max(most, Staged(rows, in, group, form).total());
    return most;
}

xnor_status launch_w4_staged(W4Kernel kernel, const void *x, long long x_stride, const float *x_scale, const void *wimg, void *y, void *workspace, int rows,
                             int in, int out, int group, int x_group, int form, int type, hipStream_t stream)
{
    const Staged st(rows, in, group, form);
    uint8_t *staged = static_cast<uint8_t *>(workspace);
    const StageArgs sa{x, x_scale, staged, x_stride, rows, in, group, x_group, x_group ? (in + x_group - 1) / x_group : 1};
    const dim3 grid((unsigned)((rows + TILE - 1) / TILE), (unsigned)((st.chunks + 3) / 4));
    if (form == ROWS_F32) w4_stage_kernel<ROWS_F32><<<grid, dim3(256), 0, stream>>>(sa);
    else if (form == ROWS_BF16) w4_stage_kernel<ROWS_BF16><<<grid, dim3(256), 0, stream>>>(sa);
    else if (form == ROWS_F16) w4_stage_kernel<ROWS_F16><<<grid, dim3(256), 0, stream>>>(sa);
    else w4_stage_kernel<ROWS_I8><<<grid, dim3(256), 0, stream>>>(sa);
    if (xnor_status e = hip_status(hipGetLastError())) return e;
    const TileArgs a{staged, static_cast<const uint8_t *>(wimg), x_scale, y, rows, in, out, type, form, st.blocks, (out + 64 * SIDE - 1) / (64 * SIDE)};
    if (kernel == W4_WAVES) {
        if (form == ROWS_I8) return x_group ? launch_waves<ROWS_I8, true>(a, group, stream) : launch_waves<ROWS_I8, false>(a, group, stream);
        if (form == ROWS_F16) return launch_waves<ROWS_F16, false>(a, group, stream);
        return launch_waves<ROWS_BF16, false>(a, group, stream);
    }
    if (form == ROWS_I8) return x_group ? launch_tiles<ROWS_I8, true>(a, group, stream) : launch_tiles<ROWS_I8, false>(a, group, stream);
    if (form == ROWS_F16) return launch_tiles<ROWS_F16, false>(a, group, stream);
    return launch_tiles<ROWS_BF16, false>(a, group, stream);
}

}  // namespace xnor
