// Products of many 8-bit rows with 8-bit weights: tiles through LDS, whole sums or shares of them that a second launch adds.
#include "xnor_internal.h"
#include "lowbit.h"
#include "tiles.h"
#include "w8_choice.h"
#include "w8_linear.h"
#include <algorithm>

namespace xnor {

namespace {

constexpr int TURNED = 32 * (64 * 4 + 16);          // bytes of 32 rows x 64 results of up to 32 bits, rows 16 bytes further apart

template <class P, bool SHARES> constexpr int lds_bytes() { return std::max(P::BUFFERS * P::BYTES, SHARES ? 0 : 12 * P::A + P::WAVES * TURNED); }

// What bounds it: 2048 rows 4096 -> 8192 in tiles of 256 x 256 78 to 83 us, 1.65 to 1.76 POP/s (a library's product to 32-bit sums 68): 58 in the chunks, of which the matrix
// instructions' 32 cycles each are 0.42 of the clock's; loads from L2 at 9 TB/s flow beside them; the rest is the launch, the first chunk's way and the results'.
// Tried: chunks of 128 and 64 bytes in 2 and 4 places (87, 98), four waves of 128 x 128 (96 to 104), operands of a step read only when it comes (91).
// SHARES: blockIdx.y of gridDim.y takes its share of the chunks and leaves its sums, 64 lanes x 4 of them in a piece, for w8_add_kernel.
template <class P, bool ALIGNED, bool SHARES> __global__ __launch_bounds__(64 * P::WAVES) void w8_tiles_kernel(W8Args a, int row_blocks, int out_blocks)
{
    constexpr int WA = P::WA, TA = P::TA, TB = P::TB;
    static_assert(TA % 2 == 0);
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    int ob, rb;
    if (!tile_of(out_blocks, row_blocks, ob, rb)) return;
    i32x16 acc[TA][TB];
    const Side w{reinterpret_cast<const uint8_t *>(a.w), (uint32_t)a.in, a.out}, x{reinterpret_cast<const uint8_t *>(a.q), (uint32_t)a.in, a.rows};
    const int chunks = (a.in + P::KB - 1) / P::KB, first = SHARES ? chunks * (int)blockIdx.y / (int)gridDim.y : 0;
    const int last = SHARES ? chunks * ((int)blockIdx.y + 1) / (int)gridDim.y : chunks;
    tile_product<Int8Op, P, ALIGNED>(acc, lds, w, x, ob * P::A, rb * P::B, first, last, a.in);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wo = wave % WA, wr = wave / WA;
    if constexpr (SHARES) {
        i32x4 *to = static_cast<i32x4 *>(a.work) + ((((size_t)blockIdx.y * row_blocks + rb) * out_blocks + ob) * P::WAVES + wave) * (TA * TB * 4 * 64) + lane;
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    to[((i * TB + j) * 4 + b) * 64] = i32x4{acc[i][j][4 * b], acc[i][j][4 * b + 1], acc[i][j][4 * b + 2], acc[i][j][4 * b + 3]};
        return;
    }
    // The outputs' scales and biases where the chunks were, and behind them a place for each wave, in which it turns 32 rows x 64 outputs so that a row's results are
    // stored next to each other (16 bytes of each of 32 rows per store: 2048 x 4096 -> 8192 81 us, 78 turned).
    float *mantissa = reinterpret_cast<float *>(lds), *bias = mantissa + P::A;
    int *exponent = reinterpret_cast<int *>(bias + P::A);
    uint8_t *turned = lds + 12 * P::A + wave * TURNED;
    __syncthreads();
    for (int i = threadIdx.x; i < P::A; i += 64 * P::WAVES) {
        const int o = min(ob * P::A + i, a.out - 1);
        const Split s(a.w_scale[o]);
        mantissa[i] = s.mantissa;
        exponent[i] = s.exponent;
        bias[i] = a.bias ? a.bias[o] : 0.0f;
    }
    __syncthreads();
    const int size = a.type == XNOR_F32 ? 4 : 2, pitch = 64 * size + 16;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int row0 = rb * P::B + (wr * TB + j) * 32;
        const Split xs(a.x_scale[min(row0 + (lane & 31), a.rows - 1)]);
#pragma unroll
        for (int pair = 0; pair < TA; pair += 2) {
#pragma unroll
            for (int i = pair; i < pair + 2; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int in_pair = (i - pair) * 32 + 8 * b + 4 * (lane >> 5), at = wo * TA * 32 + pair * 32 + in_pair;
                    const f32x4 m = *reinterpret_cast<const f32x4 *>(mantissa + at), c = *reinterpret_cast<const f32x4 *>(bias + at);
                    const i32x4 e = *reinterpret_cast<const i32x4 *>(exponent + at);
                    f32x4 y;
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = scaled_sum(acc[i][j][4 * b + k], xs, m[k], e[k]) + c[k];
                    store_four(turned + (lane & 31) * pitch, a.type, in_pair, y, 4);
                }
            // (a wave's own place: its lanes run in step, and what it writes there it reads itself)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const int o0 = ob * P::A + (wo * TA + pair) * 32, per_row = 4 * size, left = (a.out - o0) * size;       // 16-byte pieces of a row; its bytes that exist
            for (int n = lane; n < 32 * per_row; n += 64) {
                const int r = n / per_row, at = 16 * (n % per_row), row = row0 + r;
                if (row >= a.rows || at >= left) continue;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(turned + r * pitch + at);
                uint8_t *to = static_cast<uint8_t *>(a.y) + ((size_t)row * a.out + o0) * size + at;
                if (left - at >= 16) {
                    *reinterpret_cast<words4_any *>(to) = v;
                } else {
#pragma unroll
                    for (int h = 0; h < 8; ++h)
                        if (2 * h < left - at) reinterpret_cast<uint16_t *>(to)[h] = (uint16_t)(v[h / 2] >> (16 * (h & 1)));
                }
            }
            asm volatile("" ::: "memory");
        }
    }
}

// The shares of four sums per thread.
template <class P> __global__ __launch_bounds__(256) void w8_add_kernel(W8Args a, int row_blocks, int out_blocks, int shares)
{
    constexpr int PER_TILE = P::WAVES * P::TA * P::TB * 4;              // pieces of 64 lanes
    const size_t piece = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6), pieces = (size_t)row_blocks * out_blocks * PER_TILE;
    const int lane = threadIdx.x & 63;
    if (piece >= pieces) return;
    const i32x4 *from = static_cast<const i32x4 *>(a.work) + piece * 64 + lane;
    i32x4 sum = *from;
    for (int s = 1; s < shares; ++s) sum += from[(size_t)s * pieces * 64];
    const int within = (int)(piece % PER_TILE), tile = (int)(piece / PER_TILE), wave = within / (P::TA * P::TB * 4), n = within % (P::TA * P::TB * 4);
    const int b = n & 3, j = n / 4 % P::TB, i = n / 4 / P::TB;
    const int row = tile / out_blocks * P::B + (wave / P::WA * P::TB + j) * 32 + (lane & 31);
    const int o = tile % out_blocks * P::A + (wave % P::WA * P::TA + i) * 32 + 8 * b + 4 * (lane >> 5);
    if (row >= a.rows || o >= a.out) return;
    const Split xs(a.x_scale[row]);
    f32x4 y;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int at = min(o + k, a.out - 1);
        y[k] = scaled_sum(sum[k], xs, Split(a.w_scale[at])) + (a.bias ? a.bias[at] : 0.0f);
    }
    store_four(a.y, a.type, (size_t)row * a.out + o, y, a.out - o);
}

template <class P, bool ALIGNED, bool SHARES> xnor_status launch(const W8Args &a, int shares, hipStream_t stream)
{
    constexpr unsigned lds = lds_bytes<P, SHARES>();
    const int row_blocks = (a.rows + P::B - 1) / P::B, out_blocks = (a.out + P::A - 1) / P::A;
    const long long count = (long long)row_blocks * out_blocks;
    static_assert(64 * P::WAVES == 512);
    if (count > W8_MOST_TILES) return XNOR_ERR_SHAPE;
    auto kernel = w8_tiles_kernel<P, ALIGNED, SHARES>;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return XNOR_ERR_HIP;
    kernel<<<dim3((unsigned)((count + 7) / 8 * 8), (unsigned)shares), dim3(64 * P::WAVES), lds, stream>>>(a, row_blocks, out_blocks);
    if (xnor_status e = hip_status(hipGetLastError())) return e;
    if (!SHARES) return XNOR_OK;
    const long long pieces = count * (P::WAVES * P::TA * P::TB * 4);
    w8_add_kernel<P><<<dim3((unsigned)((pieces + 3) / 4)), dim3(256), 0, stream>>>(a, row_blocks, out_blocks, shares);
    return hip_status(hipGetLastError());
}

typedef TilePlan<2, 4, 4, 2, 64, 3> Large;
typedef TilePlan<2, 4, 2, 1, 128, 2> Small;
typedef TilePlan<2, 4, 2, 1, 128, 4> Deep;
static_assert(Large::A == W8_LARGE && Large::B == W8_LARGE && Small::A == W8_SMALL && Small::B == W8_SMALL);

}  // namespace

xnor_status launch_w8_tiles(const W8Args &a, int side, int shares, hipStream_t stream)
{
    const bool aligned = a.in % 16 == 0;
    if (side == W8_LARGE) return aligned ? launch<Large, true, false>(a, 1, stream) : launch<Large, false, false>(a, 1, stream);
    if (w8_alone(a.rows, a.in, a.out, shares)) return shares > 1 ? launch<Deep, true, true>(a, shares, stream) : launch<Deep, true, false>(a, 1, stream);
    if (shares > 1) return aligned ? launch<Small, true, true>(a, shares, stream) : launch<Small, false, true>(a, shares, stream);
    return aligned ? launch<Small, true, false>(a, 1, stream) : launch<Small, false, false>(a, 1, stream);
}

}  // namespace xnor
