// linear_cut.h -- how a matrix product is cut into tiles and shares of its sums
// (product.h); host code without HIP, so that it can be asked on the CPU.
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

// The same where the last tiles alone may be split: the first `whole` tiles, whole
// rounds of the GPU's 256 or 512 places for them, are done by a block each, the sums
// of the others are shared out among `splits`.  320 tiles of 256 take two rounds of
// which the second is a quarter full; split in four it takes a quarter of the time.
struct TailCut {
    int tile, whole, splits, share;  // share: steps of a split
    int64_t tail;                    // tiles that are split; 0 with splits 1
    double us;                       // the estimate
    size_t bytes() const { return splits > 1 ? (size_t)tail * splits * tile * tile * 4 : 0; }
};
// Measured with weights that come from memory, against every cut of 16 to 2048 rows: a
// step of a 128 tile takes 0.45 to 0.58 us alone on its CU and 0.95 beside another,
// times `pace`, what the kernel's steps take of those in 16 bits; beginning and end of
// a 256 tile 11; a share's values move at 8 TB/s while the caches hold them, in a
// launch of 5; shares of fewer than six steps never paid.  The choice is 1% from the
// fastest cut in the mean and 19% at worst (256 x 2048 x 4096 in bf16, 20 us for 17).
// beside: in tiles of 128 with one place of each CU, where another product has the other.
inline TailCut cut_tail(int64_t ni, int64_t nj, int64_t nr, int size, bool beside = false, double pace = 1) {
    const int64_t steps = std::max<int64_t>(1, ceil_div(nr * size, kStepBytes));
    TailCut best{};
    for (int tile = beside ? 128 : 256; tile >= 128; tile /= 2) {
        const int64_t tiles = ceil_div(ni, tile) * ceil_div(nj, tile), places = tile == 256 || beside ? 256 : 512;
        const auto time = [&](int64_t blocks, int64_t share) {
            if (blocks == 0) return 0.0;
            if (tile == 256) return ceil_div(blocks, 256) * (11 + share * (1.05 + 0.53 * std::min(1.0, blocks / 256.0)));
            return blocks <= 256 && !beside ? 3 + share * pace * (0.45 + 0.13 * blocks / 256.0) : ceil_div(blocks, places) * (5 + share * pace * 0.95);
        };
        for (int part = 0; part < 2; ++part) {
            const int64_t whole = part ? tiles / places * places : 0, tail = tiles - whole;
            if (part && (whole == 0 || tail == 0)) continue;
            for (int want = 1; want <= 8 && (want == 1 || (steps / want >= 6 && tail * want <= 2 * places)); ++want) {
                if (part && want == 1) continue;
                const int share = want == 1 ? (int)steps : (int)(ceil_div(ceil_div(steps, want), 2) * 2);
                const int splits = (int)ceil_div(steps, share);
                double us = time(whole, steps) + time(tail * splits, share);
                const double moved = splits * (double)tail * std::min<int64_t>(tile, ni) * std::min<int64_t>(tile, nj) * 8;
                if (splits > 1) us += 5 + moved / (moved < 256e6 ? 8e6 : 4e6);
                if (best.tile == 0 || us < best.us) best = TailCut{tile, (int)(splits > 1 ? whole : tiles), splits, share, splits > 1 ? tail : 0, us};
            }
        }
    }
    return best;
}

}  // namespace tg
