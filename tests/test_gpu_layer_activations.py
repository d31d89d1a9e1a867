"""Activations and their slopes over their whole range, against 64 bits."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E32, TINY, U

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def sweep(dtype):
    """z from -12 to 6 as x [n, 1], and w = [[1]]: the product is x itself, without an error."""
    z = torch.linspace(-12, 6, 4609).to(dtype)
    return z[:, None].cuda(), torch.ones(1, 1, dtype=dtype, device="cuda")


def units(z):
    """Relative error of exp(-z^2 / 2) and of what it is multiplied by: two roundings of the exponent z^2 / 2, its base's
    constant and the function itself, and 64 units for the quotient, the polynomial and the products."""
    return (1.5 * z.square() + 64) * E32


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gelu_has_its_relative_accuracy_where_it_is_small(dtype):
    x, one = sweep(dtype)
    y = layer().tg_linear(x, one, act="gelu")
    z = R.f64(x)
    want = R.act(z, "gelu")
    R.within(y, want, (1.01 * U[dtype] + units(z)) * want.abs() + TINY[dtype])


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_the_slope_of_gelu_has_the_accuracy_of_its_terms(dtype):
    x, one = sweep(dtype)
    dx, _, _ = layer().tg_linear_grad(torch.ones_like(x), x, one, pre=x, act="gelu")
    z = R.f64(x)
    want = R.slope(z, "gelu")
    # Phi(z) and z phi(z) are added: an error of either is not relative to the sum
    terms = 0.5 * torch.erfc(-z / 2 ** 0.5) + z.abs() * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    R.within(dx, want, 1.01 * U[dtype] * want.abs() + units(z) * terms + TINY[dtype])


@pytest.mark.parametrize("name", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype,big", [(F16, 400.0), (BF16, 2.0 ** 64)])
def test_a_pre_activation_beyond_the_type_has_the_slope_of_its_limit(dtype, big, name):
    """z is finite in 32 bits or in 64, `pre` rounds to an infinity: act is 0 below, its slope 0 below and 1 above."""
    L = layer()
    x = torch.tensor([[1.0, 2.0], [-big, big / 8], [big, 0.0], [0.5, -1.0]], dtype=dtype, device="cuda")
    w = torch.tensor([[big, 1.0], [0.25, -0.5]], dtype=dtype, device="cuda")
    dy = torch.tensor([[1.0, -2.0]] * 4, dtype=dtype, device="cuda")
    y, pre = L.tg_linear(x, w, act=name, keep_pre=True)
    if dtype == F16:
        assert float(pre[1, 0]) == -float("inf") and float(pre[2, 0]) == float("inf")
        assert float(y[1, 0]) == 0 and float(y[2, 0]) == float("inf")
    pre = pre.clone()
    pre[1, 0], pre[2, 0] = -float("inf"), float("inf")
    dx, dw, db = L.tg_linear_grad(dy, x, w, pre=pre, act=name, bias_grad=True)
    far = pre.clone()  # as far out as 64 bits need to have the limits exactly
    far[1, 0], far[2, 0] = -1e4, 1e4
    want = R.linear_grads(dy, x, w, far, name)
    for key, got in (("dx", dx), ("dw", dw), ("db", db)):
        R.within(got, *want[key], key)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_a_pre_activation_that_is_no_number_stays_one(name):
    L = layer()
    x = torch.ones(3, 4, dtype=BF16, device="cuda")
    pre = torch.zeros(3, 4, dtype=BF16, device="cuda")
    pre[1, 2] = float("nan")
    w = torch.eye(4, dtype=BF16, device="cuda")
    dx, _, db = L.tg_linear_grad(x, x, w, pre=pre, act=name, bias_grad=True)
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[[0, 2]]).all()
    assert torch.equal(torch.isnan(db).cpu(), torch.tensor([False, False, True, False]))
