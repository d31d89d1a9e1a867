"""How products whose last tiles are split are cut, from the rule itself compiled for the host."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
#include <cstdio>
#include "linear_cut.h"
int main() {
    long i, j, r;
    int size, beside;
    double pace;
    while (scanf("%ld %ld %ld %d %d %lf", &i, &j, &r, &size, &beside, &pace) == 6) {
        const tg::TailCut c = tg::cut_tail(i, j, r, size, beside != 0, pace);
        printf("%d %d %ld %d %d %zu\\n", c.tile, c.whole, (long)c.tail, c.splits, c.share, c.bytes());
    }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    """(tile, whole tiles, tiles that are split, splits, steps of a split, bytes) of each product."""
    place = tmp_path_factory.mktemp("cut")
    (place / "cut.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2606_16907_amd", "csrc"), "-o",
                           str(place / "cut"), str(place / "cut.cpp")])

    def ask(products):
        text = "".join("%d %d %d %d %d %g\n" % (p if len(p) == 6 else p + (1,)) for p in products)
        lines = subprocess.check_output([str(place / "cut")], input=text.encode()).decode().splitlines()
        return [tuple(int(x) for x in line.split()) for line in lines]

    return ask


def test_every_tile_and_step_is_covered_once(cut):
    sizes = [(i, j, r, size, beside, pace) for i in (0, 1, 128, 129, 1000, 5003, 20000) for j in (0, 1, 257, 4096, 28672) for r in (0, 1, 64, 65, 1000, 14336, 70000)
             for size in (1, 2) for beside in (0, 1) for pace in ((1, 1.1, 1.25, 1.4) if size == 1 and not beside else (1,))]
    for (i, j, r, size, beside, _), (tile, whole, tail, splits, share, nbytes) in zip(sizes, cut(sizes), strict=True):
        steps, tiles = max(1, -(-r * size // 128)), -(-i // tile) * -(-j // tile)
        what = (i, j, r, size, beside)
        assert tile in (128, 256) and not (beside and tile == 256), what
        assert whole + tail == tiles and (tail == 0) == (splits == 1 or tiles == 0) and 1 <= splits <= 8, what
        assert (splits - 1) * share < steps <= splits * share and (splits == 1 or share % 2 == 0), what
        assert nbytes == (tail * splits * tile * tile * 4 if splits > 1 else 0), what
        assert nbytes <= 2 * 512 * 256 * 256 * 4, what


def test_a_last_round_that_is_not_full_is_split(cut):
    """The sizes of the GPU tests and timed calls that are there for it: 320 tiles of 256 on 256 places; and the last of
    rounds that are full is not."""
    (tile, whole, tail, splits, _, _), full = cut([(5003, 4096, 14336, 1, 0), (8192, 8192, 7168, 1, 0)])
    assert (tile, whole, tail) == (256, 256, 64) and splits > 1
    assert full[2] == 0 and full[3] == 1


def test_sizes_of_the_large_tiles_take_them(cut):
    """tests/test_gpu_layer_gated.py and test_gpu_layer_blocks.py: rows, columns of the sums, r; blocks with the pace of
    either type of scales.  Each has sizes that are split, in their tail alone, and not at all."""
    gated = [(1500, 3000, 8200, 2, 0), (3500, 4082, 1000, 2, 0), (4352, 4352, 4104, 2, 0), (4352, 4352, 2048, 2, 0)]
    blocks = [(1500, 3000, 8200), (3500, 4075, 2064), (3841, 3841, 1999), (3000, 1500, 16400), (4352, 4352, 4100)]
    for sizes in (gated, [(*s, 1, 0, 1.4) for s in blocks], [(*s, 1, 0, 1.25) for s in blocks]):
        taken = cut(sizes)
        assert all(t[0] == 256 for t in taken)
        assert any(t[1] > 0 and t[3] > 1 for t in taken) and any(t[1] == 0 and t[3] > 1 for t in taken) and any(t[3] == 1 for t in taken)


def test_few_rows_are_split_by_the_rows_there_are(cut):
    """112 tiles leave more than half of the places free: 16 rows and 64 are shared out, as 16 rows of partial sums cost
    little; sums of 16 steps are not."""
    few = cut([(16, 14336, 4096, 1, 0, 1.4), (64, 14336, 4096, 1, 0, 1.25), (16, 14336, 4096, 1, 0, 1.1)])
    assert [t[3] for t in few] == [2, 2, 2]
    short, = cut([(16, 8192, 2048, 1, 0, 1.1)])
    assert short[3] == 1
