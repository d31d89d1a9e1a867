"""Plain 64-bit forms of the layer operators on the CPU, and the bounds within
which the kernels' results have to lie.

u is the largest relative error of rounding to the output's type (half a unit in
the last place), e = 2^-24 that of a 32-bit operation.
"""
import math

import torch

E4M3 = torch.float8_e4m3fn
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
E32 = 2.0 ** -24


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64)


def act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def linear(x, w, bias=None, name="none", residual=None, x_scale=None, w_scale=None):
    """(y, z, bound of z's error): the bound is that of any order of 32-bit additions of k products."""
    x, w = f64(x), f64(w)
    if x_scale is not None:
        x, w = x * f64(x_scale)[:, None], w * f64(w_scale)[:, None]
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + f64(bias), size + f64(bias).abs()
    bound = (x.shape[1] + 16) * E32 * size
    y = act(z, name)
    return (y if residual is None else y + f64(residual)), z, bound


def linear_bound(y, z, bound, dtype, residual=None):
    """act has a slope of at most 1.13 and is evaluated to a few units of 32 bits; then the sum and one rounding."""
    more = 0 if residual is None else f64(residual).abs()
    return U[dtype] * y.abs() * 1.01 + 1.2 * bound + 16 * E32 * (z.abs() + y.abs() + more) + TINY[dtype] + 1e-30


def linear_grads(dy, x, w, pre, name):
    """{name: (value, bound)}.  dz is rounded to the inputs' type, independently for each element: a sum of n such errors
    of at most u |dz w| each stays within 8 standard deviations, u / sqrt(3) of the root of the sum of squares."""
    u, tiny = U[dy.dtype], TINY[dy.dtype]
    dy, x, w, dtype = f64(dy), f64(x), f64(w), dy.dtype
    dz = dy * slope(f64(pre), name) if name != "none" else dy
    out = {}
    for key, a, b in (("dx", dz, w), ("dw", dz.t(), x)):
        v = a @ b
        n = a.shape[1]
        rounding = 0 if name == "none" else 8 / math.sqrt(3) * u * (a.square() @ b.square()).sqrt() + tiny * b.abs().sum(0)
        out[key] = v, 1.01 * u * v.abs() + rounding + (n + 32) * E32 * (a.abs() @ b.abs()) + tiny + 1e-30
    v = dz.sum(0)
    out["db"] = v, 1.01 * u * v.abs() + (dz.shape[0] + 32) * E32 * dz.abs().sum(0) + tiny + 1e-30
    return out


def within(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    far = (got - want).abs() - bound
    assert not torch.isnan(got).any(), f"{what}: NaN"
    if far.numel():
        i = int(far.argmax())
        assert far.max() <= 0, (f"{what}: {got.reshape(-1)[i].item()!r} for {want.reshape(-1)[i].item()!r}, bound "
                                f"{bound.expand_as(want).reshape(-1)[i].item():.3g}, {int((far > 0).sum())} of {far.numel()} outside")


def rows(gen, m, n, dtype, pad=0, std=1.0, offset=0):
    """[m, n] on the GPU inside rows that are `pad` wider, from `offset` elements into the buffer on."""
    flat = (torch.randn(m * (n + pad) + offset, generator=gen) * std).to(dtype).cuda()
    return flat[offset:].view(m, n + pad)[:, :n]


def generator(*key):
    gen = torch.Generator()
    gen.manual_seed(sum((i + 1) * ord(c) for i, c in enumerate(repr(key))))
    return gen
