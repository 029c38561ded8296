// Which kernel takes a weight gradient, and in how many parts its factors are.  Plain numbers, no HIP headers: a host compiler can ask which kernel a size reaches.
#pragma once
#include <algorithm>
#include <cmath>
#include "xnor_lowbit.h"

namespace xnor {

constexpr int STAGED_ROWS = 64;         // of a workgroup of the staging launch: operands are whole multiples of them
constexpr int DIRECT_SIDE = 64;         // of the kernel of few products

// A factor that is more than one float16 holds, q * scale or a float32 gradient (with scales of rows the gradient times the scale), is two of them, 22 bits.  For bfloat16 results
// q * scale and a 16-bit gradient's product with its scale are one, 11 bits, off by 2^-11 of themselves at most: an eighth of the half steps that the result (2^-8), a bfloat16
// gradient (2^-8; a float16 one's is 2^-11) and a row's codes (1 / 254 of the largest) are rounded by.  2048 rows 4096 -> 8192 in groups, bfloat16 throughout, 164 us, with two parts
// 262.  A float32 gradient carries no such rounding and keeps its bits: 277 (cut to 11 bits 174).
struct GradientParts {
    int padded, parts_x, parts_g;       // padded: rows
    bool by_row;                        // the scales are the rows'
    constexpr GradientParts(int rows, int group, int type, int w_type)
        : padded((rows + STAGED_ROWS - 1) / STAGED_ROWS * STAGED_ROWS), parts_x(w_type == XNOR_BF16 || group == 0 ? 1 : 2),
          parts_g(type == XNOR_F32 || (group == 0 && w_type != XNOR_BF16) ? 2 : 1), by_row(group == 0) {}
};

// Tiles of 256 x 256, 128 x 128 and 64 x 64 by their time in us, fitted to 75 products (1 to 8192 rows, 128 to 9216 inputs, 128 to 8192 outputs) for each number of parts: a
// chunk of 64 rows takes the way to L2 and back, or where there are more tiles what L2 gives; a large tile is alone on its CU.  2048 rows 4096 -> 8192 in bfloat16 170, 187 and
// 263 us in all; 256 rows 9216 -> 4096 65, 52, 85; 2048 rows 1024 -> 1024 78, 42, 31, with float32 results 124, 50, 35.
struct GradientChoice {
    bool direct;        // the kernel of few products, otherwise tiles of this side
    int side;
    double time;        // of the tiles' launch
};
inline GradientChoice gradient_tiles(const GradientParts &p, int in, int out, int w_bytes)
{
    const double chunks = p.padded / 64.0, kept = 2e-7 * in * out * w_bytes;
    auto tiles = [&](int side) { return std::ceil((double)in / side) * std::ceil((double)out / side); };
    const int parts = p.parts_x + p.parts_g;
    const double small = chunks * (parts == 2   ? std::max(0.33, 0.00131 * tiles(64))
                                   : parts == 3 ? std::max(0.5, 0.0018 * tiles(64))
                                                : std::max(0.65, 0.0019 * tiles(64)));
    const double middle = chunks * (parts == 2   ? std::max(0.6, 0.0023 * tiles(128))
                                    : parts == 3 ? std::max(1.0, 0.0038 * tiles(128))
                                                 : std::max(1.55, 0.0055 * tiles(128)));
    const double rounds = std::ceil(tiles(256) / 256), large = rounds * (parts == 2 ? 1.6 * chunks + 10 : 3.3 * chunks + 13);
    if (parts < 4 && large < std::min(small, middle) + kept) return {false, 256, large};
    return middle < small ? GradientChoice{false, 128, middle} : GradientChoice{false, 64, small};
}

// The direct kernel by its time in us, fitted likewise; the others' range, staging and launches take 13 and their way through memory.  2 rows 371 -> 2011 bfloat16 4.5 and
// 12, 64 rows 1003 -> 1000 float32 6.4 and 15, 256 rows 1024 -> 1024 bfloat16 11 and 17, 777 rows 1003 -> 1000 float32 25 and 27; 2048 rows 512 -> 512 bfloat16 52 and 23, 64 rows
// 4096 -> 4096 84 and 25.  Over 70 products (1 to 1156 rows, 17 to 2900 inputs and outputs) the choice takes 1.001 of the faster one's time.
inline bool gradient_direct_is_faster(const GradientParts &p, int rows, int in, int out, const GradientChoice &staged)
{
    if (in < 2 || out < 2) return false;
    const double rounds = std::ceil(std::ceil(in / 64.0) * std::ceil(out / 64.0) / 256), bytes = 2.0 * p.padded * ((double)in * p.parts_x + (double)out * p.parts_g);
    return 2 + rounds * (2.8 + 0.0235 * rows) < 13 + staged.time + bytes / 3.5e6;
}
inline GradientChoice gradient_choice(const GradientParts &p, int rows, int in, int out, int w_bytes)
{
    GradientChoice c = gradient_tiles(p, in, out, w_bytes);
    c.direct = gradient_direct_is_faster(p, rows, in, out, c);
    return c;
}

}  // namespace xnor
