// linear_cut.h -- how a matrix product is cut into tiles and shares of its sums
// (linear.hip); host code without HIP, so that it can be asked on the CPU.
#pragma once

#include <algorithm>
#include <cstdint>

#include "sizes.h"

namespace tg {

constexpr int kStepBytes = 128;  // of r in a step of the loop over it

// How a product is cut: tiles of 256 or 128, and r into splits, whichever is
// estimated to take the least time.  Measured, in us: a step of a 256 tile takes
// 1.05 while few of the 256 CUs work and 1.58 when all do, one of a 128 tile 0.38
// to 0.56 alone on its CU and 0.95 beside another; beginning and end of a tile
// take 9 and 3 to 5; the shares of a split are written and read at 4 TB/s, at 8
// while the caches hold them, in a launch of 3.  2048 x 1024 x 4096: 24 in tiles
// of 128 and 36 of 256; 4096^3: 125 of 128 and 110 of 256; its gradient with sums
// of 4096 over 2048 x 1024: 34 unsplit, 29 in two.  Tiles of 256 x 128 were within
// 5% of the better of the two.  The epilogue's operands are not counted: with them
// and unaligned rows a short product takes up to twice the estimate, in either tile.
struct Cut {
    int tile, splits, share;  // share: steps of a split
};
inline Cut cut_product(int64_t ni, int64_t nj, int64_t nr, int size) {
    const int64_t steps = std::max<int64_t>(1, ceil_div(nr * size, kStepBytes));
    Cut best{256, 1, (int)steps};
    double least = 0;
    for (int tile = 256; tile >= 128; tile /= 2) {
        for (int want = 1; want <= 8 && (want == 1 || (steps / want >= 4 && ni * nj <= 1 << 26)); ++want) {
            const int share = want == 1 ? (int)steps : (int)(ceil_div(ceil_div(steps, want), 2) * 2);
            const int splits = (int)ceil_div(steps, share);
            const int64_t blocks = ceil_div(ni, tile) * ceil_div(nj, tile) * splits;
            const double used = std::min(1.0, blocks / 256.0);
            double us;
            if (tile == 256)
                us = ceil_div(blocks, 256) * (9 + share * (1.05 + 0.53 * used));
            else
                us = blocks <= 256 ? 3 + share * (0.33 + 0.23 * used) : ceil_div(blocks, 512) * (5 + share * 0.95);
            const double moved = splits * (double)ni * nj * 8;
            if (splits > 1) us += 3 + moved / (moved < 64e6 ? 8e6 : 4e6);
            if (least == 0 || us < least) least = us, best = Cut{tile, splits, share};
        }
    }
    return best;
}

}  // namespace tg
