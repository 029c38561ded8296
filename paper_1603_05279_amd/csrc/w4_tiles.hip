// Products of many rows with 4-bit weights: rows staged once as operands, then tiles of 128 outputs x 128 rows.
#include "xnor_internal.h"
#include "lowbit.h"
#include "w4_form.h"
#include "w4_image.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr int TILE = 16, BLOCK = 8;         // rows or outputs of a matrix instruction, such tiles of a workgroup's side
constexpr int SPLIT_CHUNKS = 4;             // a share of the inputs is a multiple of 4 chunks: whole quads of groups

// What the rows become (the first kernel writes it, the second reads it), in a workspace of the caller's:
//   operands  [block of 128 rows][chunk of 128 inputs][part][tile of 16 rows][step][lane][16 bytes]: 16 bits, 4 steps of 32 inputs; 8 bits, 2 steps
//             of 64.  Tiles past the last row are not written: they meet no result that is kept
//   sums      [tile of 16 rows][quad of groups][lane][16 bytes], 16 bits only: the groups' sums of x as three bfloat16 numbers in an order that
//             gives all products with a second factor's three but the smallest: lane 16 i + r is row r, group i of the quad
//   scales    [tile of 16 rows][group][row] float32, 8-bit rows with scales of groups only
//   partial   [share][row][out, whole tiles] float32, where the inputs are shared out
struct Staged {
    int blocks, chunks, parts, groups, quads;
    bool bytes;
    __host__ __device__ Staged(int rows, int in, int group, int form)
        : blocks((rows + TILE * BLOCK - 1) / (TILE * BLOCK)), chunks((in + 127) / 128), parts(form == ROWS_F32 ? 3 : 1),
          groups((in + group - 1) / group), quads(form == ROWS_I8 ? 0 : (groups + 3) / 4), bytes(form == ROWS_I8) {}
    __host__ __device__ int tile_bytes() const { return bytes ? 2048 : 4096; }
    __host__ __device__ size_t sums_at() const { return (size_t)blocks * chunks * parts * BLOCK * tile_bytes(); }
    __host__ __device__ size_t scales_at() const { return sums_at() + (size_t)blocks * BLOCK * quads * 1024; }
    __host__ __device__ size_t partial_at() const { return scales_at() + (bytes ? (size_t)blocks * BLOCK * groups * 64 : 0); }
};

// x cut off to three bfloat16 numbers whose sum it is (an infinity has no rest)
__device__ __forceinline__ void three_parts(float x, uint32_t *p)
{
    const bool finite = __builtin_fabsf(x) < __builtin_inff();
    p[0] = (__float_as_uint(x) | (x != x ? 0x00400000u : 0u)) >> 16;
    const float rest = finite ? x - __uint_as_float(p[0] << 16) : 0.0f;
    p[1] = __float_as_uint(rest) >> 16;
    p[2] = __float_as_uint(rest - __uint_as_float(p[1] << 16)) >> 16;
}

struct StageArgs {
    const void *x;
    const float *x_scale;
    uint8_t *staged;
    long long x_stride;
    int rows, in, group, x_group, x_groups;
};

// A wave stages 16 rows x 128 inputs; what bounds it: memory.
template <int X>
__global__ __launch_bounds__(256) void w4_stage_kernel(StageArgs a)
{
    typedef Form<X> F;
    const Staged st(a.rows, a.in, a.group, X);
    const int lane = threadIdx.x & 63, r = lane & 15, quarter = lane >> 4;
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6), tile = blockIdx.y;
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
            for (int i = 0; i < 8; ++i) s += v[j].v[i];
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
        u32x4 *sums = reinterpret_cast<u32x4 *>(a.staged + st.sums_at()) + (size_t)tile * st.quads * 64;
        const int last = chunk == st.chunks - 1 ? 4 * st.quads : first + per_chunk;
        for (int g = first + quarter; g < last; g += 4) {
            const int i = g - first;
            uint32_t p[3];
            three_parts(i >= per_chunk ? 0.0f : i == 0 ? sum[0] : i == 1 ? sum[1] : i == 2 ? sum[2] : sum[3], p);
            sums[(size_t)(g >> 2) * 64 + (g & 3) * 16 + r] = u32x4{p[0] | p[1] << 16, p[0] | p[1] << 16, p[2] | p[0] << 16, p[2] | p[1] << 16};
        }
    }
}

struct TileArgs {
    const uint8_t *staged, *image;
    const float *x_scale;
    float *partial;
    void *y;
    int rows, in, out, group, type, form;
    int row_blocks, out_blocks, shares, per_share;      // chunks of a share
};

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(1))) uint8_t global_u8;

__device__ __forceinline__ void to_lds(const uint8_t *from, uint8_t *to)        // 16 bytes per lane, to + 16 * lane
{
    __builtin_amdgcn_global_load_lds((global_u8 *)from, (lds_u8 *)to, 16, 0, 0);
}

// STEPS of 32 inputs per group.  Four waves, each 64 outputs x 64 rows.  The rows' operands of a chunk and the weights' scales go straight to LDS while the
// chunk before is multiplied (two buffers, one barrier per chunk); the codes go to the registers of the lanes that multiply them.
// GROUPED: 8-bit rows with scales of groups.
template <int X, int STEPS, bool GROUPED>
__global__ __launch_bounds__(256, 2) void w4_tiles_kernel(TileArgs a)
{
    typedef Form<X> F;
    constexpr int TB = X == ROWS_I8 ? 2048 : 4096, PER_CHUNK = 4 / STEPS;
    constexpr int FACTORS = BLOCK * PER_CHUNK * 64;                              // bytes of the scales of a chunk
    constexpr int ZEROS = X == ROWS_I8 ? BLOCK * PER_CHUNK * 16 : 0;              // and of the zero points, where the sums are exact
    constexpr int BUFFER = BLOCK * TB + FACTORS * (GROUPED ? 2 : 1) + ZEROS;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const W4Layout l(a.out, a.in, a.group);
    const Staged st(a.rows, a.in, a.group, a.form);
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wo = wave & 1, wr = wave >> 1;
    // workgroups go to the XCDs in turn: each takes a run of neighbouring tiles
    const int count = a.row_blocks * a.out_blocks * a.shares, per_xcd = (count + 7) / 8;
    const int id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || id >= count) return;
    const int share = id / (a.row_blocks * a.out_blocks), rest = id % (a.row_blocks * a.out_blocks);
    const int rb = rest % a.row_blocks, ob = rest / a.row_blocks;
    const int otile = ob * BLOCK + wo * 4, rtile = rb * BLOCK + wr * 4;
    const int first = share * a.per_share, last = min(first + a.per_share, l.chunks);
    const int parts = st.parts;

    const u32x4 *codes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[i] = reinterpret_cast<const u32x4 *>(a.image) + (size_t)min(otile + i, l.tiles - 1) * l.chunks * 64 + lane;
    const uint8_t *scales = a.image + l.scale_at();
    const uint8_t *rows_from = a.staged + (size_t)rb * st.chunks * parts * BLOCK * TB;
    // chunk c (parts of it one after another: step = chunk * parts + part)
    auto fetch_rows = [&](int step, int buffer) {
        const uint8_t *from = rows_from + (size_t)step * BLOCK * TB + tid * 16;
        uint8_t *to = lds + buffer * BUFFER + wave * 1024;
#pragma unroll
        for (int i = 0; i < BLOCK * TB / 4096; ++i) to_lds(from + i * 4096, to + i * 4096);
        // scales: lane = tile, group of the chunk, quarter; a group past the last meets sums of zero
        const int chunk = step / parts;
        if (X == ROWS_I8 && wave == 3 && lane < BLOCK * PER_CHUNK) {
            const int g = min(chunk * PER_CHUNK + lane % PER_CHUNK, l.groups - 1);
            to_lds(a.image + l.zero_at() + ((size_t)min(ob * BLOCK + lane / PER_CHUNK, l.tiles - 1) * l.groups + g) * 16, lds + buffer * BUFFER + BUFFER - ZEROS);
        }
        if (wave * 64 < BLOCK * PER_CHUNK * 4) {
            const int f = tid, tile = f / (PER_CHUNK * 4), g = min(chunk * PER_CHUNK + f / 4 % PER_CHUNK, l.groups - 1);
            if (f < BLOCK * PER_CHUNK * 4) {
                const size_t o = ((size_t)min(ob * BLOCK + tile, l.tiles - 1) * l.groups + g) * 64 + (f & 3) * 16;
                to_lds(scales + o, lds + buffer * BUFFER + BLOCK * TB + wave * 1024);
            }
            if (GROUPED && f < BLOCK * PER_CHUNK * 4) {
                const size_t o = ((size_t)(rb * BLOCK + tile) * l.groups + g) * 64 + (f & 3) * 16;
                to_lds(a.staged + st.scales_at() + o, lds + buffer * BUFFER + BLOCK * TB + FACTORS + wave * 1024);
            }
        }
    };
    f32x4 total[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) total[i][j] = f32x4{0, 0, 0, 0};
    u32x4 w[4], next[4];
    const int steps = (last - first) * parts;
    fetch_rows(first * parts, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = codes[i][(size_t)first * 64];
    for (int s = 0; s < steps; ++s) {
        const int buffer = s & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                            // (the buffer is filled, the other one is read no more)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = next[i];
        if (s + 1 < steps) {
            fetch_rows(first * parts + s + 1, buffer ^ 1);
            const int chunk = first + (s + 1) / parts;
#pragma unroll
            for (int i = 0; i < 4; ++i) next[i] = codes[i][(size_t)chunk * 64];
        }
        const uint8_t *x = lds + buffer * BUFFER + wr * 4 * TB + lane * 16;
        const uint8_t *sw = lds + buffer * BUFFER + BLOCK * TB + wo * 4 * PER_CHUNK * 64 + quarter * 16;
        const uint8_t *sx = lds + buffer * BUFFER + BLOCK * TB + FACTORS + wr * 4 * PER_CHUNK * 64 + col * 4;
        const uint8_t *zero = lds + buffer * BUFFER + BUFFER - ZEROS + wo * 4 * PER_CHUNK * 16 + col;
        // one tile of outputs after the other, so that the scaling of one meets the products of the next
        constexpr int LOADS = TB / 1024;
        u32x4 b[LOADS][4];
#pragma unroll
        for (int t = 0; t < LOADS; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) b[t][j] = *reinterpret_cast<const u32x4 *>(x + j * TB + t * 1024);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typename F::acc_t acc[4];
            uint32_t z = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (t % STEPS == 0) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = typename F::acc_t{0, 0, 0, 0};
                    if (X == ROWS_I8) z = zero[(i * PER_CHUNK + t / STEPS) * 16] * 0x01010101u;
                }
                if constexpr (X != ROWS_I8) {
                    const auto wide = F::widen(w[i][t]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = F::mfma(wide, b[t][j], acc[j]);
                } else if constexpr (STEPS == 1) {          // (two groups in the 64 inputs of an instruction)
                    const long wide = F::widen(w[i][t], z);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[j] = F::mfma(wide, (long)((uint64_t)b[t / 2][j][2 * (t & 1)] | (uint64_t)b[t / 2][j][2 * (t & 1) + 1] << 32), acc[j]);
                } else if (t % 2 == 0) {
                    const uint32_t c0 = w[i][t], c1 = w[i][t + 1];
                    const i32x4 wide{(int)F::minus(c0, z), (int)F::minus(c0 >> 4, z), (int)F::minus(c1, z), (int)F::minus(c1 >> 4, z)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wide, __builtin_bit_cast(i32x4, b[t / 2][j]), acc[j], 0, 0, 0);
                }
                if (t % STEPS != STEPS - 1) continue;
                const int g = t / STEPS;
                const f32x4 f = *reinterpret_cast<const f32x4 *>(sw + (i * PER_CHUNK + g) * 64);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float c = GROUPED ? *reinterpret_cast<const float *>(sx + (j * PER_CHUNK + g) * 64) : 1.0f;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float part = (float)acc[j][v];
                        if (GROUPED) part *= c;
                        total[i][j][v] = __builtin_fmaf(f[v], part, total[i][j][v]);
                    }
                }
            }
        }
    }
    // what the offset and the zero points add is taken out: - scale (OFFSET + zero) times the groups' sums, four groups per instruction, both
    // factors as three bfloat16 numbers (all products but the smallest: 2^-32 of the largest)
    const uint8_t *zeros = a.image + l.zero_at();
    const int quad_end = min((last * PER_CHUNK + 3) / 4, st.quads);         // (none for 8 bits)
    for (int quad = first * PER_CHUNK / 4; quad < quad_end; ++quad) {
        bf16x8 b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            b[j] = __builtin_bit_cast(bf16x8, reinterpret_cast<const u32x4 *>(a.staged + st.sums_at())[((size_t)(rtile + j) * st.quads + quad) * 64 + lane]);
        const int g = min(4 * quad + quarter, l.groups - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t f = ((size_t)min(otile + i, l.tiles - 1) * l.groups + g) * 16 + col;
            uint32_t p[3];
            three_parts(-(reinterpret_cast<const float *>(scales)[f] * (16.0f + (float)zeros[f])), p);
            const u32x4 k{p[0] | p[0] << 16, p[1] | p[1] << 16, p[0] | p[2] << 16, p[1] | p[2] << 16};
#pragma unroll
            for (int j = 0; j < 4; ++j) total[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), b[j], total[i][j], 0, 0, 0);
        }
    }
    const int pitch = l.tiles * TILE;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = (rtile + j) * TILE + col;
        if (row >= a.rows) continue;
        if (a.shares > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (otile + i < l.tiles)
                    *reinterpret_cast<f32x4 *>(a.partial + ((size_t)share * a.rows + row) * pitch + (otile + i) * TILE + 4 * quarter) = total[i][j];
            continue;
        }
        const float c = X == ROWS_I8 && !GROUPED ? a.x_scale[row] : 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int o = (otile + i) * TILE + 4 * quarter;
            f32x4 v = total[i][j];
            if (X == ROWS_I8 && !GROUPED) v *= c;
            store_four(a.y, a.type, (size_t)row * a.out + o, v, a.out - o);
        }
    }
}

// The shares of a result added in their order.
__global__ __launch_bounds__(256) void w4_join_kernel(const float *partial, const float *row_scale, void *y, int rows, int out, int shares, int type)
{
    const int pitch = (out + TILE - 1) / TILE * TILE, quads = pitch / 4;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)rows * quads) return;
    const size_t row = i / quads;
    const int o = (int)(i % quads) * 4;
    f32x4 v{0, 0, 0, 0};
    for (int s = 0; s < shares; ++s) v += *reinterpret_cast<const f32x4 *>(partial + ((size_t)s * rows + row) * pitch + o);
    if (row_scale) v *= row_scale[row];
    store_four(y, type, row * out + o, v, out - o);
}

struct Shares {
    int count, chunks;
};
// Shares of the inputs: until there are two workgroups per CU.
Shares shares_of(int rows, int in, int out)
{
    const int chunks = (in + 127) / 128, longest = (chunks + SPLIT_CHUNKS - 1) / SPLIT_CHUNKS;
    const long long tiles = (long long)((rows + 127) / 128) * ((out + 127) / 128);
    const int want = (int)std::max<long long>(1, std::min<long long>({512 / tiles, longest, 16}));
    const int per = (longest + want - 1) / want * SPLIT_CHUNKS;
    return {(chunks + per - 1) / per, per};
}

template <int X, bool GROUPED> xnor_status launch_tiles(const TileArgs &a, hipStream_t stream)
{
    const int tb = X == ROWS_I8 ? 2048 : 4096, factors = BLOCK * (128 / a.group) * (64 * (GROUPED ? 2 : 1) + (X == ROWS_I8 ? 16 : 0));
    const unsigned lds = 2 * (BLOCK * tb + factors);
    const long long count = (long long)a.row_blocks * a.out_blocks * a.shares;
    if (count > 0x7fffff00 / 256) return XNOR_ERR_SHAPE;
    const dim3 grid((unsigned)((count + 7) / 8 * 8));
    auto go = [&](auto kernel) {
        if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
            return XNOR_ERR_HIP;
        kernel<<<grid, dim3(256), lds, stream>>>(a);
        return hip_status(hipGetLastError());
    };
    if (a.group == 32) return go(w4_tiles_kernel<X, 1, GROUPED>);
    if (a.group == 64) return go(w4_tiles_kernel<X, 2, GROUPED>);
    return go(w4_tiles_kernel<X, 4, GROUPED>);
}

}  // namespace

bool w4_tiles_applies(int rows) { return rows > 64; }

size_t w4_tiles_workspace_bytes(int rows, int in, int out, int group)
{
    const Shares s = shares_of(rows, in, out);
    const size_t partial = s.count > 1 ? (size_t)s.count * rows * ((out + TILE - 1) / TILE * TILE) * sizeof(float) : 0;
    return std::max(Staged(rows, in, group, ROWS_F32).partial_at(), Staged(rows, in, group, ROWS_I8).partial_at()) + partial;
}

xnor_status launch_w4_tiles(const void *x, long long x_stride, const float *x_scale, const void *wimg, void *y, void *workspace, int rows, int in, int out,
                            int group, int x_group, int form, int type, hipStream_t stream)
{
    const Staged st(rows, in, group, form);
    const Shares s = shares_of(rows, in, out);
    uint8_t *staged = static_cast<uint8_t *>(workspace);
    const StageArgs sa{x, x_scale, staged, x_stride, rows, in, group, x_group, x_group ? (in + x_group - 1) / x_group : 1};
    const dim3 grid((unsigned)((st.chunks + 3) / 4), (unsigned)((rows + TILE - 1) / TILE));
    if (form == ROWS_F32) w4_stage_kernel<ROWS_F32><<<grid, dim3(256), 0, stream>>>(sa);
    else if (form == ROWS_BF16) w4_stage_kernel<ROWS_BF16><<<grid, dim3(256), 0, stream>>>(sa);
    else if (form == ROWS_F16) w4_stage_kernel<ROWS_F16><<<grid, dim3(256), 0, stream>>>(sa);
    else w4_stage_kernel<ROWS_I8><<<grid, dim3(256), 0, stream>>>(sa);
    if (xnor_status e = hip_status(hipGetLastError())) return e;
    const TileArgs a{staged, static_cast<const uint8_t *>(wimg), x_scale, reinterpret_cast<float *>(staged + st.partial_at()), y, rows, in, out, group,
                     type, form, st.blocks, (out + TILE * BLOCK - 1) / (TILE * BLOCK), s.count, s.chunks};
    xnor_status e;
    if (form == ROWS_I8) e = x_group ? launch_tiles<ROWS_I8, true>(a, stream) : launch_tiles<ROWS_I8, false>(a, stream);
    else if (form == ROWS_F16) e = launch_tiles<ROWS_F16, false>(a, stream);
    else e = launch_tiles<ROWS_BF16, false>(a, stream);
    if (e != XNOR_OK || s.count == 1) return e;
    const size_t quads = (size_t)rows * ((out + TILE - 1) / TILE * 4);
    w4_join_kernel<<<dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream>>>(a.partial, form == ROWS_I8 && !x_group ? x_scale : nullptr, y, rows, out,
                                                                                    s.count, type);
    return hip_status(hipGetLastError());
}

}  // namespace xnor
