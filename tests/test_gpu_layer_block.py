"""The operators together: a feed-forward block as it trains and answers, and the command that measures it."""
import pytest
import torch

from tests import layer_ref as R

pytestmark = pytest.mark.gpu


def block(hidden=192, ffn=328, act="gelu", bits=32):
    from paper_2606_16907_amd.measure_layer import FeedForward
    return FeedForward(hidden, ffn, act, bits, seed=3)


def inputs(rows, hidden):
    gen = R.generator("block", rows, hidden)
    return [R.rows(gen, rows, hidden, torch.bfloat16) for _ in range(3)]


def plain(layer, x, residual, dout, pre):
    """The block in 64 bits by autograd, from the bf16 weights.  relu's slope jumps at 0, so it is taken on the side on
    which the block's own z lies: a z within its rounding of 0 may lie on either."""
    ws = [R.f64(p).requires_grad_() for p in layer.params]
    norm, up, up_bias, down, down_bias = ws
    h = (R.f64(x) + R.f64(residual)).requires_grad_()
    y = h / (h.square().mean(1, keepdim=True) + layer.eps).sqrt() * norm
    z = y @ up.t() + up_bias
    a = z * (R.f64(pre) > 0) if layer.act == "relu" else R.act(z, layer.act)
    out = a @ down.t() + down_bias + h
    out.backward(R.f64(dout))
    return out.detach(), h.grad, [w.grad for w in ws]


def near(got, want, what, tol):
    """Relative 2-norm of the difference: each of some dozen roundings to 8 bits of mantissa in a row is off by at most
    2^-8, 0.4 of that in the mean, independently of the others; 5 times the root of their number covers them."""
    far = float((R.f64(got) - want).norm() / want.norm())
    assert far < tol, (what, far)


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_block_against_autograd(act):
    layer = block(act=act)
    x, residual, dout = inputs(70, 192)
    out, kept = layer.forward(x, residual)
    dx = layer.backward(dout, kept)
    want_out, want_dx, want_grads = plain(layer, x, residual, dout, kept[2])
    tol = 5 * 12 ** 0.5 * 0.4 * 2.0 ** -8
    near(out, want_out, "out", tol)
    near(dx, want_dx, "dx", tol)
    for k, (g, w) in enumerate(zip(layer.grads, want_grads)):
        near(g, w, f"gradient {k}", tol)


@pytest.mark.parametrize("bits", [32, 8])
def test_training_lowers_the_loss(bits):
    layer = block(bits=bits)
    x, residual, target = inputs(256, 192)
    losses = []
    for _ in range(60):
        out, kept = layer.forward(x, residual)
        dout = (out.float() - target.float()) / out.numel() * 2
        losses.append(float((out.float() - target.float()).square().mean()))
        layer.backward((dout * 256).to(torch.bfloat16), kept)
        layer.step(lr=3e-3, weight_decay=0.0)
    assert losses[-1] < 0.6 * losses[0], (losses[0], losses[-1])
    assert all(bool(torch.isfinite(p.float()).all()) for p in layer.params)


def test_answer_in_8_bits_follows_the_forward_pass():
    layer = block(256, 512)
    x, residual, _ = inputs(5, 256)
    out, _ = layer.forward(x, residual)
    got = layer.answer(x, residual, layer.eight_bits())
    # e4m3 is off by 2^-4 at most, 2^-5.3 in the mean, in both operands of a product whose terms are independent
    near(got, R.f64(out), "answer", 2 * 2 ** 0.5 * 2.0 ** -5.3)


def test_command():
    from paper_2606_16907_amd import measure_layer
    m = measure_layer.main(["--hidden", "256", "--ffn", "512", "--seq", "128", "--steps", "2"])
    assert m["rows"] == 128 and m["parameters"] == 2 * 256 * 512 + 2 * 256 + 512
    assert 0 < m["eta"] < 1 and abs(m["bytes_per_parameter"] - 16) < 1e-9
    assert m["plan_s_measured_eta"] > m["plan_s_eta_1"] > 0
    assert abs(measure_layer.measure(256, 512, 128, bits=8, steps=2)["bytes_per_parameter"] - 10.03) < 0.2
