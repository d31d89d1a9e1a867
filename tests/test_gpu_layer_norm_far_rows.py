"""Gradients of layer norms whose rows lie so far from zero that a mean over its rstd leaves 32 bits."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E32, TINY, U

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FAR, RSTD = 2.0 ** 120, 316.0  # their product is 4.2e38; a constant row's rstd at an eps of 1e-5


def layer():
    from paper_2606_16907_amd import layer as L
    return L


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 64), (19, 64), (3, 100), (70, 100), (19, 523), (5, 777), (19, 1027), (19, 1549), (19, 2057), (19, 4111), (5, 8203),
                                       (19, 12297), (3, 16391), (5, 33001), (3, 70001)])
def test_constant_rows(rows, cols, dtype):
    """h - mean is 0 in every column, so dx = rstd (g - mean(g)) and dweight = 0: nothing of the elements that a last unit
    has past the row's end, nor of threads that have none, may reach the row's sums.  A mean over n terms is off by
    (n / 64 + 24) e of the mean size, as the kernels add at most n / 64 of them, and 24 more, in a row."""
    gen = R.generator("far rows", rows, cols, dtype)
    w, dy = (1 + R.rows(gen, 1, cols, F32)[0] * 0.2).to(dtype), R.rows(gen, rows, cols, dtype, 3)
    sign = 1.0 - 2.0 * (torch.arange(rows, device="cuda") % 2)
    h = (FAR * sign).to(dtype)[:, None].expand(rows, cols).contiguous()
    rstd = torch.full((rows,), RSTD, device="cuda")
    dx, dw, db = layer().tg_layer_norm_grad(dy, h, w, FAR * sign, rstd)
    d = R.f64(dy)
    g = d * R.f64(w)
    mean = g.mean(1, keepdim=True)
    want = RSTD * (g - mean)
    err = RSTD * ((cols / 64 + 24) * E32 * g.abs().mean(1, keepdim=True) + 8 * E32 * (g.abs() + mean.abs()))
    R.within(dx, want, 1.01 * U[dtype] * want.abs() + 2 * err + TINY[dtype], "dx")
    assert bool((dw == 0).all())
    R.within(db, d.sum(0), 1.01 * U[dtype] * d.sum(0).abs() + (rows + 16) * E32 * d.abs().sum(0) + TINY[dtype], "dbias")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_forward_and_backward(dtype):
    """64 columns, whose sum is exact: the forward pass gives the mean and rstd itself."""
    L, gen = layer(), R.generator("far both", dtype)
    x, w = torch.full((9, 64), FAR, device="cuda", dtype=dtype), torch.ones(64, device="cuda", dtype=dtype)
    dy = R.rows(gen, 9, 64, dtype)
    f = L.tg_layer_norm(x, w, eps=1e-5)
    assert bool((f.mean == FAR).all()) and bool((f.y == 0).all())
    dx = L.tg_layer_norm_grad(dy, f.hidden, w, f.mean, f.rstd)[0]
    g = R.f64(dy)
    want = (g - g.mean(1, keepdim=True)) * 1e-5 ** -0.5
    R.within(dx, want, 1.01 * U[dtype] * want.abs() + 64 * E32 * 1e-5 ** -0.5 * g.abs().amax(1, keepdim=True), "dx")
