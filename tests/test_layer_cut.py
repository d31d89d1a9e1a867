"""How products are cut, from the rule itself compiled for the host: the sizes of the tests of large tiles must take them."""
import os
import subprocess

import pytest

from tests import layer_tiles as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
#include <cstdio>
#include "linear_cut.h"
int main() {
    long i, j, r;
    int size;
    while (scanf("%ld %ld %ld %d", &i, &j, &r, &size) == 4) {
        const tg::Cut c = tg::cut_product(i, j, r, size);
        printf("%d %d %d\\n", c.tile, c.splits, c.share);
    }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    """(tile, splits, steps of a split) of each product (rows, columns, length of the sums, bytes of an element)."""
    place = tmp_path_factory.mktemp("cut")
    (place / "cut.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2606_16907_amd", "csrc"), "-o",
                           str(place / "cut"), str(place / "cut.cpp")])

    def ask(products):
        text = "".join(f"{i} {j} {r} {size}\n" for i, j, r, size in products)
        lines = subprocess.check_output([str(place / "cut")], input=text.encode()).decode().splitlines()
        return [tuple(int(x) for x in line.split()) for line in lines]

    return ask


def test_sizes_of_the_large_tiles_take_them(cut):
    products = list(S.products())
    for (i, j, r, size, shared), (tile, splits, _) in zip(products, cut([p[:4] for p in products]), strict=True):
        assert tile == 256 and (splits > 1) == shared, (i, j, r, size)


def test_some_of_them_take_several_turns_of_the_steady_loop(cut):
    """Two steps a turn, while more than six whole ones are left."""
    for size in (1, 2):
        whole = [r * size // 128 for _, _, r, s, shared in S.products() if s == size and not shared]
        assert sum(w >= 12 for w in whole) >= 2 and min(whole) < 6


@pytest.mark.parametrize("size", [1, 2])
def test_shares_cover_the_sums_in_pairs_of_steps(cut, size):
    sizes = [(i, j, r, size) for i in (1, 128, 129, 1000, 5000) for j in (1, 257, 4096) for r in (0, 1, 64, 65, 1000, 4097, 70000)]
    for (i, j, r, _), (tile, splits, share) in zip(sizes, cut(sizes), strict=True):
        steps = max(1, -(-r * size // 128))
        assert tile in (128, 256) and (splits - 1) * share < steps <= splits * share, (i, j, r)
        assert splits == 1 or share % 2 == 0, (i, j, r)
