"""Plain 64-bit forms of the gated projections and their bounds, in the manner of layer_ref."""
import math

from tests import layer_ref as R
from tests.layer_ref import E32, TINY, U

def dropped(a, b):
    """What the 8-bit matrix instruction drops of a @ b.t(), in 64 bits.  It adds products in groups of eight consecutive ones
    and cuts each off, towards 0, at 2^-13 of the power of two in the largest (with 448 * 448 - 448 * 448 in a group a product
    of 7 is lost and one of 8 stays, with 256 and 16 in the place of 448 the same numbers times 2^0 and 2^-8).  The largest
    itself has 8 bits and stays.  So up to seven products of a group lose up to u = 2^-13 of its largest, m: that is at most
    7 u m in one group, and in many, where signs are random, 8 standard deviations, 1 / sqrt(3) of the root of the sum over
    groups of 7 (u m)^2; the sum of m^2 is at most that of all squares, and 8 sqrt(7 / 3) is more than 7."""
    return 8 * (7 / 3) ** 0.5 * 2.0 ** -13 * (a.square() @ b.square().t()).sqrt()

def projections(x, w_gate, w_up, gate_bias, up_bias, x_scale=None, gate_scale=None, up_scale=None):
    """((gate, bound), (up, bound)) of any order of 32-bit additions, with scales also of products in 8 bits."""
    out = []
    for w, b, s in ((w_gate, gate_bias, gate_scale), (w_up, up_bias, up_scale)):
        _, z, bound = R.linear(x, w, b, x_scale=x_scale, w_scale=s)
        if x_scale is not None:
            bound = bound + dropped(R.f64(x) * R.f64(x_scale)[:, None], R.f64(w) * R.f64(s)[:, None])
        out.append((z, bound))
    return out

def forward(gate, up, name, dtype):
    """(y, bound): act has a slope of at most 1.13 and is evaluated to a few units of 32 bits; then one product, one rounding."""
    (g, bg), (u, bu) = gate, up
    value = R.act(g, name)
    bv = 1.13 * bg + 16 * E32 * (g.abs() + value.abs())
    y = value * u
    return y, 1.01 * U[dtype] * y.abs() + 1.01 * (bv * (u.abs() + bu) + value.abs() * bu) + 4 * E32 * y.abs() + TINY[dtype] + 1e-30

def kept(z, bound, dtype):
    return z, 1.01 * U[dtype] * z.abs() + 1.01 * bound + TINY[dtype]

def grads(dy, x, w_gate, w_up, gate, up, name):
    """{key: (value, bound)} from gate and up as they are kept.  dgate and dup are rounded to the inputs' type, independently
    for each element: a sum of such errors, of at most u |d w| each, stays within 8 standard deviations, u / sqrt(3) of the
    root of the sum of squares.  The slope and the activation are evaluated to 16 units of 32 bits of 1 + |gate|."""
    u, tiny, dtype = U[dy.dtype], TINY[dy.dtype], dy.dtype
    dy, x, w_gate, w_up, gate, up = (R.f64(t) for t in (dy, x, w_gate, w_up, gate, up))
    dg, du = dy * up * R.slope(gate, name), dy * R.act(gate, name)
    ag, au = (dy * up).abs() * (1 + gate.abs()), dy.abs() * (1 + gate.abs())
    out = {}

    def add(key, pairs, n):
        v = sum(a @ b for a, b, _ in pairs)
        squares = sum(a.square() @ b.square() for a, b, _ in pairs)
        size = sum(a.abs() @ b.abs() for a, b, _ in pairs)
        evaluated = sum(16 * E32 * s @ b.abs() for _, b, s in pairs)
        lost = sum(tiny * b.abs().sum(0) for _, b, _ in pairs)
        out[key] = v, (1.01 * u * v.abs() + 8 / math.sqrt(3) * u * squares.sqrt() + lost + (n + 32) * E32 * size + evaluated + tiny + 1e-30)

    m, n = dy.shape
    add("dx", ((dg, w_gate, ag), (du, w_up, au)), 2 * n)
    add("dw_gate", ((dg.t(), x, ag.t()),), m)
    add("dw_up", ((du.t(), x, au.t()),), m)
    for key, d, s in (("dgate_bias", dg, ag), ("dup_bias", du, au)):
        v = d.sum(0)
        out[key] = v, 1.01 * u * v.abs() + (m + 32) * E32 * d.abs().sum(0) + 16 * E32 * s.sum(0) + tiny + 1e-30
    return out
