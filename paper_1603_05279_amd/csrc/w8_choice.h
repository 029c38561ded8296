// Which kernel takes a product of 8-bit rows with 8-bit weights.  Plain numbers, no HIP headers: a host compiler can ask which kernel a size reaches.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstddef>

namespace xnor {

constexpr int W8_LARGE = 256, W8_SMALL = 128;           // sides of the tiles of w8_tiles.hip
constexpr long long W8_MOST_TILES = 0xffffff00LL / 512;    // of a launch, whose threads are counted in 32 bits

// The shortest of their times in us, fitted to 150 products (inputs 256 to 9216, outputs 256 to 8192, 1 to 2048 rows, half of them no multiple of
// anything).
struct W8Choice {
    int tiles, side, shares;        // w8_rows_kernel's row tiles, or the side of w8_tiles.hip's tiles and the shares of the inputs
    double time;
};

inline double w8_blocks(int n, int side) { return std::ceil((double)n / side); }

// w8_rows_kernel reads every weight once per 16, 32 or 64 rows and splits the inputs over its waves.  One, two and four tiles: 16 rows 9216 -> 4096 10.6, 11.5, 13.6; 32 rows
// 4096 -> 4096 10.0, 8.1, 9.2; 64 rows 17, 13.5, 11.7 (128 x 128 in four shares 15).  Rows that start between words of 32 bits: 15 rows 6086 -> 7076 31 (in shares 24).
inline W8Choice w8_by_rows(int rows, int in, int out)
{
    const double turns = std::ceil(std::ceil(in / 128.0) / 8);
    W8Choice best{0, 0, 1, 0.0};
    for (int tiles : {1, 2, 4}) {
        const double n = w8_blocks(out, 16) * w8_blocks(rows, 16 * tiles) / 256;
        const double time = 4.3 + (tiles == 1 ? 0.85 : tiles == 2 ? 1.2 : 2.05) * (in % 4 ? 2.4 : 1.0) * turns * std::max(n, 0.7);
        if (best.tiles == 0 || time < best.time) best = {tiles, 0, 1, time};
    }
    return best;
}
// Tiles of 128 x 128: what a CU gets out of L2 bounds a chunk, 0.65 us for 256 workgroups (12 TB/s), and its way there and back where there are fewer.  In shares of the inputs
// where that fills the chip, which costs another launch and the sums' way through memory.  256 rows 9216 -> 4096 in 1, 2, 3, 4 and 6 shares 39, 26, 24, 26, 28; 512 rows
// 4096 -> 4096 in 1 and 2 21, 25.
inline W8Choice w8_by_small_tiles(int row_blocks, int in, int out)
{
    const double chunks = std::ceil(in / 128.0), tiles = (double)row_blocks * w8_blocks(out, W8_SMALL);
    W8Choice best{0, W8_SMALL, 0, 0.0};
    for (int shares : {1, 2, 3, 4, 6, 8}) {
        const double n = tiles * shares / 256;
        if (shares > 1 && (n > 2 || chunks < 2 * shares)) break;
        const double chunk = in % 16 == 0 ? std::max(0.48, 0.65 * n) : in % 4 == 0 ? std::max(0.85, 0.85 * n) : std::max(1.25, 0.95 * n);
        const double time = 4.0 + chunk * std::ceil(chunks / shares) + (shares > 1 ? 2.5 + 0.026 * tiles * shares : 0.0) + 0.002 * tiles;
        if (best.shares == 0 || time < best.time) best = {0, W8_SMALL, shares, time};
    }
    return best;
}
// Tiles of 256 x 256 take half as much out of L2 per result, one workgroup to a CU.  2048 rows 4096 -> 8192 83 us, in tiles of 128 x 128 91; 4096 rows 158, 175; 1024 rows 70, 45.
inline W8Choice w8_by_large_tiles(int rows, int in, int out)
{
    const double tiles = w8_blocks(rows, W8_LARGE) * w8_blocks(out, W8_LARGE), rounds = std::ceil(tiles / 256);
    return {0, W8_LARGE, 1, 12 + (tiles <= 128 ? 0.85 : 1.06) * std::ceil(in / 64.0) * rounds * (in % 4 ? 1.5 : in % 16 ? 1.3 : 1.0) + 0.012 * tiles};
}
inline W8Choice w8_choice(int rows, int in, int out)
{
    W8Choice best = w8_by_rows(rows, in, out);
    const W8Choice small = w8_by_small_tiles((int)w8_blocks(rows, W8_SMALL), in, out), large = w8_by_large_tiles(rows, in, out);
    if (small.time < best.time && w8_blocks(rows, W8_SMALL) * w8_blocks(out, W8_SMALL) <= W8_MOST_TILES) best = small;
    if (large.time < best.time) best = large;
    return best;
}
// Bytes of the shares' sums: the most of any number of rows up to this one.  (More than 256 tiles are not shared.)
inline size_t w8_share_bytes(int rows, int in, int out)
{
    size_t most = 0;
    for (int b = 1; b <= (int)w8_blocks(rows, W8_SMALL) && b * w8_blocks(out, W8_SMALL) <= 256; ++b) {
        const int shares = w8_by_small_tiles(b, in, out).shares;
        if (shares > 1) most = std::max(most, (size_t)shares * b * (size_t)w8_blocks(out, W8_SMALL) * W8_SMALL * W8_SMALL * 4);
    }
    return most;
}
// Whether a tile of 128 x 128 is alone on its CU, where four chunks in LDS are faster than two (256 x 4096 -> 4096 20 us, with two 23); from 256 workgroups on two of them share a CU
// and its loads better (512 x 4096 -> 8192 27, 29).  Of rows of whole 16 bytes.
inline bool w8_alone(int rows, int in, int out, int shares) { return in % 16 == 0 && w8_blocks(rows, W8_SMALL) * w8_blocks(out, W8_SMALL) * shares <= 192; }

}  // namespace xnor
