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

// Rows of x up to which product_few is faster than tiles, with two weights or scaled
// blocks, each with `columns` sums in all and rows of row_bytes.  Up to 16 it reads as
// much: 16 rows through 7168 x 4096 take 12.6 us with scaled blocks and 11.5 gated in 8
// bits, in tiles 17.5 and 17.2; through 4096 x 14336 23 and 21, in tiles 23 and 19; from
// 100 MB on 12 rows (16384 x 16384: 75 for 75, 16 rows 84 for 76).  Up to 8192 columns
// tiles are few and split, which is another launch: 32 rows through 7168 x 4096 take
// 15.8 for 17.9, through 4096 x 4096 10.3 for 16.8, 64 rows through 2048 x 2048 9.8 for
// 19.2; longer rows are slower (64 through 7168 x 2048: 20.3 for 19.4).
inline int64_t few_rows(int64_t columns, int64_t row_bytes) {
    const int64_t all = columns * row_bytes;
    if (columns <= 8192 && row_bytes <= 4096 && all <= 17000000) return 64;
    if (columns <= 8192 && row_bytes <= 8192 && all <= 30000000) return 32;
    return all <= 100000000 ? 16 : 12;
}
// The same where an operand would have to be packed first.  Rows at multiples of 4 bytes
// are read as fast as others: 48 through 7169 x 7169 take 39 us for 44, 32 through 4097 x
// 20002 43 for 62 (48 of gated operands 57 for 51), 32 through 16385 x 4098 50 for 53, of
// gated ones 50 for 47, 24 42 for 46; 64 through 40966 bytes x 512 24 for 41.  Over 198
// sizes the limits are 0.1% from the faster of both in the mean and 5% at worst.  Rows
// that are not, the slower the longer: 4098 x 289 up to some 38 rows (32 take 17 us for
// 19, 48 22 for 20), 10486 x 2289 up to some 14 (8 take 24 for 29, 24 37 for 29), 8190 x
// 16390 up to fewer than 8 (111 for 89).
inline int64_t few_packed_rows(int64_t columns, int64_t row_bytes, bool words) {
    const int64_t all = std::max<int64_t>(1, columns * row_bytes);
    if (words) return all <= 25000000 ? 64 : row_bytes > 16384 ? 24 : all <= 60000000 ? 48 : 32;
    const int64_t most = std::min(130000 / std::max<int64_t>(1, row_bytes), 2 + 500000000 / all);
    return std::max<int64_t>(1, std::min<int64_t>(64, most));
}

// The gradients of two weights' products: dx [m, k] with sums over r, and dw [rows, k]
// with sums over m; either may be left out.  Both in one launch (`two`), in tiles of 128
// with a place on each CU, where the longer of them is estimated to take less than they
// do one after the other.
struct GradCut {
    TailCut dx, dw;
    bool two;
};
inline GradCut cut_gradients(int64_t m, int64_t k, int64_t r, int64_t rows, bool dx, bool dw) {
    GradCut c{};
    if (dx) c.dx = cut_tail(m, k, r, 2);
    if (dw) c.dw = cut_tail(rows, k, m, 2);
    if (!dx || !dw) return c;
    const TailCut a = cut_tail(m, k, r, 2, true), b = cut_tail(rows, k, m, 2, true);
    // a grid holds fewer than 2^32 threads, 256 a block
    c.two = std::max(a.us, b.us) < c.dx.us + c.dw.us && a.whole + a.tail * a.splits + b.whole + b.tail * b.splits < (1 << 24);
    if (c.two) c.dx = a, c.dw = b;
    return c;
}

}  // namespace tg
