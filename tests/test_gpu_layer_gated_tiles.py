"""The gated projections in 8 bits and the weights' gradients in the tiles and shares that large calls take, against 64 bits."""
import ctypes

import pytest
import torch

from tests import gated_ref as G
from tests import gated_tiles as S
from tests import layer_ref as R
from tests.layer_ref import E4M3

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def quantised(t, pad=0):
    scale = (t.abs().amax(1) / 448).clamp_min(1e-12)
    wide = torch.full((t.shape[0], t.shape[1] + pad), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3)  # NaN past the rows
    wide[:, :t.shape[1]] = (t / scale[:, None]).to(E4M3)
    return wide[:, :t.shape[1]], scale


@pytest.mark.parametrize("pad", [0, 3, 16])
@pytest.mark.parametrize("m,k,n", list(S.EIGHT_BITS))
def test_forward_in_8_bits(m, k, n, pad):
    gen = R.generator("gated8 tiles", m, k, n, pad)
    out, name = (BF16, "silu") if pad else (F16, "gelu")
    x, sx = quantised(R.rows(gen, m, k, F32), pad)
    (wg, sg), (wu, su) = (quantised(R.rows(gen, n, k, F32, std=k ** -0.5), pad) for _ in range(2))
    bg, bu = ([R.rows(gen, 1, n, out, std=0.5)[0] for _ in range(2)]) if pad else (None, None)
    y, gate, up = layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act=name, x_scale=sx, gate_scale=sg, up_scale=su, out_dtype=out, keep_pre=True)
    want = G.projections(x, wg, wu, bg, bu, sx, sg, su)
    R.within(gate, *G.kept(*want[0], out), "gate")
    R.within(up, *G.kept(*want[1], out), "up")
    R.within(y, *G.forward(*want, name, out), "y")
    again = layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act=name, x_scale=sx, gate_scale=sg, up_scale=su, out_dtype=out)
    assert torch.equal(y, again)


def operands(gen, m, k, n):
    pad = 3 if k % 2 else 0
    x, wg, wu = R.rows(gen, m, k, BF16, pad), R.rows(gen, n, k, BF16, 0, k ** -0.5), R.rows(gen, n, k, BF16, pad, k ** -0.5)
    dy, gate, up = (R.rows(gen, m, n, BF16, p) for p in (0, pad, 8))
    return dy, x, wg, wu, gate, up


@pytest.mark.parametrize("m,k,n", list(S.GRADIENTS) + [s for s in S.ONE_LAUNCH if s not in S.GRADIENTS])
def test_gradients(m, k, n):
    args = operands(R.generator("gated grad tiles", m, k, n), m, k, n)
    got = layer().tg_gated_grad(*args, act="silu", bias_grad=True)
    want = G.grads(*args, "silu")
    for key, value in want.items():
        R.within(getattr(got, key), *value, key)
    assert all(torch.equal(a, b) for a, b in zip(got, layer().tg_gated_grad(*args, act="silu", bias_grad=True), strict=True))


@pytest.mark.parametrize("m,k,n", list(S.WEIGHTS))
def test_gradients_of_the_weights(m, k, n):
    args = operands(R.generator("gated weights", m, k, n), m, k, n)
    got, want = layer().tg_gated_grad(*args, act="gelu", x_grad=False), G.grads(*args, "gelu")
    for key in ("dw_gate", "dw_up"):
        R.within(getattr(got, key), *want[key], key)


@pytest.mark.parametrize("which", ["dw_gate", "dw_up"])
@pytest.mark.parametrize("m,k,n", list(S.ONE_WEIGHT))
def test_gradient_of_one_weight(m, k, n, which):
    """Through the C entry, which allows it; nothing past the output's rows is written."""
    L = layer()
    args = operands(R.generator("gated one weight", m, k, n), m, k, n)
    place = torch.full((n + 128, k), 7.0, dtype=BF16, device="cuda")
    lds = [t.stride(0) for t in args]  # dy, x, w_gate, w_up, gate, up
    dy, x, wg, wu, gate, up = (t.data_ptr() for t in args)
    outs = {key: place.data_ptr() if key == which else None for key in ("dw_gate", "dw_up")}
    a = L.TgGatedGradArgs(dy, gate, up, x, wg, wu, None, outs["dw_gate"], outs["dw_up"], None, None, m, n, k, lds[0], lds[4], lds[5], lds[1], lds[2], lds[3],
                          k, k, k, 1, L.ACTS["silu"])
    lib = L.load_library()
    ws = torch.empty(lib.tg_gated_grad_workspace_bytes(a), dtype=torch.uint8, device="cuda")
    assert lib.tg_gated_grad(ctypes.byref(a), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    R.within(place[:n], *G.grads(*args, "silu")[which], which)
    assert bool((place[n:] == 7).all())
