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
