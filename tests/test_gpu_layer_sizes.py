"""Matrix products of a million rows, whose outputs pass 2^35 elements, against 64 bits at sampled rows and columns."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E32, U

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_a_million_rows_by_32768_columns():
    from paper_2606_16907_amd import layer as L
    m, k, n = 1 << 20, 64, 1 << 15
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.randn(m, k, generator=gen, device="cuda").to(BF16)
    w = (torch.randn(n, k, generator=gen, device="cuda") / 8).to(BF16)
    y = L.tg_linear(x, w)
    rows, cols = torch.tensor([0, 1, 127, 77777, m // 2, m - 129, m - 1]), torch.tensor([0, 63, 12345, n - 1])
    want, z, bound = R.linear(x[rows], w)
    R.within(y[rows], want, R.linear_bound(want, z, bound, BF16), "y")
    dx, dw, db = L.tg_linear_grad(y, x, w, bias_grad=True)
    for got, a, b in ((dx[rows], R.f64(y[rows]), R.f64(w)), (dw[cols], R.f64(y[:, cols]).t(), R.f64(x))):
        v, size = a @ b, a.abs() @ b.abs()
        R.within(got, v, 1.01 * U[BF16] * v.abs() + (a.shape[1] + 32) * E32 * size + 1e-30)
    v, size = R.f64(y[:, cols]).sum(0), R.f64(y[:, cols]).abs().sum(0)
    R.within(db[cols], v, 1.01 * U[BF16] * v.abs() + (m + 32) * E32 * size, "db")
    del x, y, dx
    torch.cuda.empty_cache()
