// Products of two matrices whose rows run along the sum, A B^T: tiles through LDS for the matrix instructions of 32 x 32 results and 32 bytes along the sum
// (8-bit integers: 32 terms, float16: 16).
#pragma once
#include "w8_form.h"

namespace xnor {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Int8Op {
    typedef i32x16 acc_t;
    static __device__ __forceinline__ acc_t mfma(i32x4 a, i32x4 b, acc_t c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};
struct HalfOp {
    typedef f32x16 acc_t;
    static __device__ __forceinline__ acc_t mfma(i32x4 a, i32x4 b, acc_t c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(1))) uint8_t global_u8;

// One side of the product: rows of `bytes`, `pitch` apart; a row's second part is `part` bytes behind its first.
struct Side {
    const uint8_t *rows;
    uint32_t pitch;
    int count;
    uint32_t part = 0;
};

// WA x WB waves, each TA x TB tiles of 32 x 32; BUFFERS chunks in LDS; a row's value is the sum of PA or PB parts, of whose products that of the second ones is left out.
template <int WA_, int WB_, int TA_, int TB_, int KB_, int BUFFERS_, int PA_ = 1, int PB_ = 1> struct TilePlan {
    static constexpr int PA = PA_, PB = PB_;
    static constexpr int WA = WA_, WB = WB_, TA = TA_, TB = TB_, KB = KB_, BUFFERS = BUFFERS_;         // KB: bytes of a row in a chunk
    static constexpr int WAVES = WA * WB, A = WA * TA * 32, B = WB * TB * 32;          // rows of a workgroup's tile
    static constexpr int BYTES = (PA * A + PB * B) * KB, LOADS = BYTES / 1024 / WAVES;  // of a chunk; 1 KB loads of a wave
    static_assert(A * KB / 1024 % WAVES == 0 && B * KB / 1024 % WAVES == 0 && PA <= 2 && PB <= 2);
};

static __device__ const __attribute__((aligned(16))) uint8_t nothing[16] = {};          // what stands behind a row's last byte

// The sums of a tile over chunks first .. last - 1 of its rows: rows a0 .. of `a`, b0 .. of `b` (past the last: the last once more, results nobody keeps).  Chunks go straight to one of BUFFERS places in LDS,
// BUFFERS - 1 chunks ahead, one barrier per chunk; a wave waits for its own loads of the oldest chunk alone.  The operands of a step are read while the matrix instructions of the step before run, across the barrier too.
// EXACT: rows are whole chunks.  ALIGNED: rows start at multiples of 16 bytes and are whole pieces of 16; others go through registers, where what is behind their end becomes 0.
// A row's 16-byte pieces lie in LDS in an order that its number turns, so that the 16 neighbouring lanes that read together (256 bytes, 64 banks) meet each bank once.
template <class Op, class P, bool ALIGNED, bool EXACT = false>
__device__ __forceinline__ void tile_product(typename Op::acc_t (&acc)[P::TA][P::TB], uint8_t *lds, const Side &a, const Side &b, int a0, int b0, int first, int last, int bytes)
{
    constexpr int WA = P::WA, TA = P::TA, TB = P::TB, KB = P::KB, STEPS = KB / 32, PIECES = KB / 16, AHEAD = P::BUFFERS - 1;
    constexpr int PA = P::PA, PB = P::PB, PART_A = P::A * KB / 1024 / P::WAVES, PART_B = P::B * KB / 1024 / P::WAVES, LOADS_A = PA * PART_A;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa = wave % WA, wb = wave / WA;
    auto turn = [](int row) { return KB == 64 ? row >> 2 & 3 : row >> 1 & 7; };
    const uint8_t *a_from = a.rows + (size_t)a0 * a.pitch, *b_from = b.rows + (size_t)b0 * b.pitch;
    uint32_t off[P::LOADS];
    int piece[P::LOADS];
#pragma unroll
    for (int i = 0; i < P::LOADS; ++i) {
        const bool is_a = i < LOADS_A;
        const int part = is_a ? i / PART_A : (i - LOADS_A) / PART_B, n = is_a ? i % PART_A : (i - LOADS_A) % PART_B;
        const int r = (n * P::WAVES + wave) * (64 / PIECES) + lane / PIECES;
        piece[i] = 16 * ((lane & (PIECES - 1)) ^ turn(r));
        off[i] = (uint32_t)min(r, (is_a ? a.count - a0 : b.count - b0) - 1) * (is_a ? a.pitch : b.pitch) + part * (is_a ? a.part : b.part) + piece[i];
    }
    i32x4 held[ALIGNED ? 1 : P::LOADS];
    // a chunk's loads, a share of them with every step (all at once they are in the way of the operands: 74.5 us for 2048 rows 4096 -> 8192 of 8 bits, so 70.6); what is not
    // whole or aligned comes with the first
    auto fetch = [&](auto surely, int c, int place, int step) {              // surely: the chunk is whole
        uint8_t *to = lds + place * P::BYTES + wave * 1024;
        const uint8_t *a_here = a_from + (size_t)c * KB, *b_here = b_from + (size_t)c * KB;
        const bool whole = surely() || (c + 1) * KB <= bytes;
        if constexpr (!ALIGNED) {
            if (step) return;
            if (whole) {
#pragma unroll
                for (int i = 0; i < P::LOADS; ++i) held[i] = *reinterpret_cast<const i32x4_any *>((i < LOADS_A ? a_here : b_here) + off[i]);
            } else {
#pragma unroll
                for (int i = 0; i < P::LOADS; ++i)
                    held[i] = bytes16(reinterpret_cast<const int8_t *>((i < LOADS_A ? a_here : b_here) + off[i] - piece[i]), piece[i], bytes - c * KB);
            }
        } else if (whole) {
#pragma unroll
            for (int i = 0; i < P::LOADS; ++i)
                if (i * STEPS / P::LOADS == step)
                    __builtin_amdgcn_global_load_lds((global_u8 *)((i < LOADS_A ? a_here : b_here) + off[i]), (lds_u8 *)(to + i * P::WAVES * 1024), 16, 0, 0);
        } else if (step == 0) {
#pragma unroll
            for (int i = 0; i < P::LOADS; ++i) {
                const uint8_t *p = c * KB + piece[i] < bytes ? (i < LOADS_A ? a_here : b_here) + off[i] : nothing;
                __builtin_amdgcn_global_load_lds((global_u8 *)p, (lds_u8 *)(to + i * P::WAVES * 1024), 16, 0, 0);
            }
        }
    };
    auto put = [&](int place) {
        if constexpr (!ALIGNED)
#pragma unroll
            for (int i = 0; i < P::LOADS; ++i) *reinterpret_cast<i32x4 *>(lds + place * P::BYTES + (i * P::WAVES + wave) * 1024 + 16 * lane) = held[i];
    };
    // a lane's operand of a step: row lane & 31 of a tile, piece 2 step + (lane >> 5)
    const int a_row = (wa * TA * 32 + (lane & 31)) * KB, b_row = (PA * P::A + wb * TB * 32 + (lane & 31)) * KB;
    i32x4 av[2][PA][TA], bv[2][PB][TB];
    auto read = [&](int place, int step) {
        const uint8_t *here = lds + place * P::BYTES + 16 * ((2 * step + (lane >> 5)) ^ turn(lane));
#pragma unroll
        for (int p = 0; p < PA; ++p)
#pragma unroll
            for (int i = 0; i < TA; ++i) av[step & 1][p][i] = *reinterpret_cast<const i32x4 *>(here + a_row + (32 * i + p * P::A) * KB);
#pragma unroll
        for (int p = 0; p < PB; ++p)
#pragma unroll
            for (int j = 0; j < TB; ++j) bv[step & 1][p][j] = *reinterpret_cast<const i32x4 *>(here + b_row + (32 * j + p * P::B) * KB);
    };
    auto multiply = [&](int step) {
#pragma unroll
        for (int p = 0; p < PA + PB - 1; ++p)                  // (first x first, second x first, first x second)
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    acc[i][j] = Op::mfma(av[step & 1][p == 1 && PA == 2 ? 1 : 0][i], bv[step & 1][p == PA && PB == 2 ? 1 : 0][j], acc[i][j]);
    };
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0;
#pragma unroll
    for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int i = 0; i < TA; ++i) av[(STEPS - 1) & 1][p][i] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int j = 0; j < TB; ++j) bv[(STEPS - 1) & 1][p][j] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) fetch(std::bool_constant<EXACT>(), min(first + i, last - 1), i, s);
        put(i);
    }
    int place = 0, c = first;
    auto turn_over = [&](auto surely) {
        // this chunk is there, everybody's part of it; and nobody reads the place of the chunk before any more
        if (ALIGNED) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * P::LOADS) : "memory");
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(place, 0);
        const int free = place == 0 ? AHEAD : place - 1, next = min(c + AHEAD, last - 1);         // (past the end: the last chunk once more, which nobody reads)
        fetch(surely, next, free, 0);
        multiply(STEPS - 1);                    // of the chunk before (the first time: zeros)
#pragma unroll
        for (int s = 1; s < STEPS; ++s) {
            read(place, s);
            fetch(surely, next, free, s);
            multiply(s - 1);
        }
        put(free);
        __builtin_amdgcn_s_waitcnt(0xc07f);                           // lgkmcnt(0): its reads of the place are over at the next barrier
        asm volatile("" ::: "memory");
        place = place == AHEAD ? 0 : place + 1;
    };
    // (whether a chunk is whole is asked only where it may not be: a branch in every step takes 3 us of those 70)
    for (const int whole = EXACT ? last : bytes / KB; c < last && min(c + AHEAD, last - 1) < whole; ++c) turn_over(std::true_type());
    if (!EXACT)
        for (; c < last; ++c) turn_over(std::false_type());
    multiply(STEPS - 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // (the loads past the end are into this workgroup's LDS)
}

// Workgroups go to the XCDs in turn: each takes a run of neighbouring tiles, in strips of `STRIP` blocks of b.  False: a workgroup without a tile.
// (At most 2^26 of them: launches of 64 threads and more reach no further.)
__device__ __forceinline__ bool tile_of(int blocks_a, int blocks_b, int &ba, int &bb)
{
    constexpr int STRIP = 4;
    const int count = blocks_a * blocks_b, per_xcd = (count + 7) / 8, id = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || id >= count) return false;
    const int strip = id / (STRIP * blocks_a), within = id - strip * STRIP * blocks_a, high = min(STRIP, blocks_b - strip * STRIP);
    ba = within / high;
    bb = strip * STRIP + within - ba * high;
    return true;
}

}  // namespace xnor
