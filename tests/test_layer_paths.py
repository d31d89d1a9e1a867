"""Which kernels the sizes of the GPU tests and of the figures in comments are done by, from the rules themselves compiled
for the host: a rule that moves would leave a test's path to no test."""
import os
import subprocess

import pytest

from tests import gated_tiles as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
#include <cstdio>
#include <cstring>
#include "linear_cut.h"
static void show(const tg::TailCut &c) { printf("%d %d %ld %d %d ", c.tile, c.whole, (long)c.tail, c.splits, c.share); }
int main() {
    char what[16];
    long a, b, c, d, e, f;
    while (scanf("%15s %ld %ld %ld %ld %ld %ld", what, &a, &b, &c, &d, &e, &f) == 7) {
        if (!strcmp(what, "few")) printf("%ld", (long)tg::few_rows(a, b));
        if (!strcmp(what, "packed")) printf("%ld", (long)tg::few_packed_rows(a, b, c != 0));
        if (!strcmp(what, "forward")) show(tg::cut_tail(a, b, c, 1, false, 1.1));
        if (!strcmp(what, "gradients")) {
            const tg::GradCut g = tg::cut_gradients(a, b, c, d, e != 0, f != 0);
            show(g.dx), show(g.dw), printf("%d", (int)g.two);
        }
        printf("\\n");
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    place = tmp_path_factory.mktemp("paths")
    (place / "paths.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2606_16907_amd", "csrc"), "-o",
                           str(place / "paths"), str(place / "paths.cpp")])

    def call(what, *numbers):
        text = what + " " + " ".join(str(int(n)) for n in (*numbers, *[0] * (6 - len(numbers)))) + "\n"
        return [int(x) for x in subprocess.check_output([str(place / "paths")], input=text.encode()).decode().split()]

    return call


def split(cut):
    """(tile, which of its tiles are split) of tile, whole tiles, split ones, splits, steps of a split."""
    return cut[0], "none" if cut[3] == 1 else "all" if cut[1] == 0 else "last"


def half(n):
    return -(-n // 64) * 64


@pytest.mark.parametrize("size", list(S.EIGHT_BITS))
def test_gated_projections_in_8_bits(ask, size):
    m, k, n = size
    assert split(ask("forward", m, 2 * n, k)) == S.EIGHT_BITS[size]
    assert m > 64, "product_few has no part in it"


@pytest.mark.parametrize("size", list(S.GRADIENTS))
def test_gradients_by_launches_of_their_own(ask, size):
    m, k, n = size
    g = ask("gradients", m, k, 2 * half(n), 2 * half(n), 1, 1)
    assert g[-1] == 0 and split(g[5:10]) == S.GRADIENTS[size]


@pytest.mark.parametrize("size", list(S.WEIGHTS))
def test_gradients_of_the_weights(ask, size):
    m, k, n = size
    g = ask("gradients", m, k, 2 * half(n), 2 * half(n), 0, 1)
    assert g[-1] == 0 and split(g[5:10]) == S.WEIGHTS[size]


@pytest.mark.parametrize("size", list(S.ONE_WEIGHT))
def test_gradient_of_one_weight(ask, size):
    m, k, n = size
    g = ask("gradients", m, k, 2 * half(n), half(n), 0, 1)
    assert g[-1] == 0 and split(g[5:10]) == S.ONE_WEIGHT[size]


@pytest.mark.parametrize("size", list(S.ONE_LAUNCH))
def test_gradients_in_one_launch(ask, size):
    m, k, n = size
    g = ask("gradients", m, k, 2 * half(n), 2 * half(n), 1, 1)
    assert g[-1] == 1 and (split(g[:5])[1], split(g[5:10])[1]) == S.ONE_LAUNCH[size]
    if size == (300, 264, 520):  # a share of dx's sums goes from one weight to the other
        assert any(s < half(n) // 64 < s + g[4] for s in range(0, 2 * half(n) // 64, g[4]))


# m, columns of the sums, bytes of a row, through product_few or not: tests/test_gpu_layer_gated.py and test_gpu_layer_blocks.py,
# and the figures beside the rule
FEW = [(1, 28672, 8192, True), (16, 10000, 8192, True), (24, 9000, 4096, False), (48, 400, 4096, True), (16, 4096, 7168, True), (12, 16384, 16384, True),
       (16, 16384, 16384, False), (32, 4096, 7168, True), (32, 4096, 4096, True), (64, 2048, 2048, True), (64, 2048, 7168, False)]


@pytest.mark.parametrize("m,columns,row_bytes,few", FEW)
def test_few_rows(ask, m, columns, row_bytes, few):
    assert (m <= ask("few", columns, row_bytes)[0]) == few


# rows whose operands would have to be packed first: columns of the sums, bytes of a row, whether rows start at multiples of 4
# bytes, rows up to which product_few measured as fast or faster, and the least number of rows from which it was 6% slower
PACKED = [(7169, 7169, True, 48, 64), (20002, 4097, True, 32, 64), (4098, 16385, True, 24, 48), (2048, 32770, True, 24, 32), (3584, 14338, True, 48, 65),
          (8194, 16382, True, 32, 48), (512, 40966, True, 64, 65), (8193, 2049, True, 64, 65), (289, 4098, False, 31, 48), (2289, 10486, False, 8, 24),
          (16390, 8190, False, 1, 8), (16390, 8191, False, 1, 8)]


@pytest.mark.parametrize("columns,row_bytes,words,faster,slower", PACKED)
def test_few_rows_that_would_be_packed(ask, columns, row_bytes, words, faster, slower):
    assert faster <= ask("packed", columns, row_bytes, words)[0] < slower
