"""The operators together in layers that are gated or have a layer norm: as they train and answer, and the command."""
import pytest
import torch

from tests import layer_ref as R
from tests.test_gpu_layer_block import inputs, near

pytestmark = pytest.mark.gpu
FORMS = [(True, "rms"), (True, "layer"), (False, "layer")]


def block(hidden=192, ffn=328, act="silu", bits=32, gated=True, norm="rms"):
    from paper_2606_16907_amd.measure_layer import FeedForward
    layer = FeedForward(hidden, ffn, act, bits, seed=3, gated=gated, norm=norm)
    gen = R.generator("biases", hidden, ffn)
    for name in ("up_bias", "down_bias", "gate_bias", "norm_bias"):  # zero at the start of training
        if hasattr(layer, name):
            t = getattr(layer, name)
            t.copy_(torch.randn(t.shape, generator=gen) * 0.2)
    return layer


def plain(layer, x, residual, dout):
    """The block in 64 bits by autograd, from the bf16 weights."""
    w = {name: R.f64(getattr(layer, name)).requires_grad_() for name in layer.grad}
    h = (R.f64(x) + R.f64(residual)).requires_grad_()
    centred = h - h.mean(1, keepdim=True) if layer.layer_norm else h
    y = centred / (centred.square().mean(1, keepdim=True) + layer.eps).sqrt() * w["norm"]
    if layer.layer_norm:
        y = y + w["norm_bias"]
    up = y @ w["up"].t() + w["up_bias"]
    a = R.act(y @ w["gate"].t() + w["gate_bias"], layer.act) * up if layer.gated else R.act(up, layer.act)
    out = a @ w["down"].t() + w["down_bias"] + h
    out.backward(R.f64(dout))
    return out.detach(), h.grad, {name: t.grad for name, t in w.items()}


@pytest.mark.parametrize("gated,norm", FORMS)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_block_against_autograd(gated, norm, act):
    layer = block(act=act, gated=gated, norm=norm)
    x, residual, dout = inputs(70, 192)
    out, kept = layer.forward(x, residual)
    dx = layer.backward(dout, kept)
    want_out, want_dx, want = plain(layer, x, residual, dout)
    # some 16 roundings to 8 bits of mantissa in a row, as `near` counts them
    tol = 5 * 16 ** 0.5 * 0.4 * 2.0 ** -8
    near(out, want_out, "out", tol)
    near(dx, want_dx, "dx", tol)
    for name, grad in layer.grad.items():
        near(grad, want[name], name, tol)


@pytest.mark.parametrize("gated,norm", FORMS)
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_run_and_replay(gated, norm, bits):
    """A training step captured in a graph gives what the same step gives eagerly."""
    layer, other = (block(gated=gated, norm=norm, bits=bits) for _ in range(2))
    x, residual, dout = inputs(64, 192)

    def work(l):
        out, kept = l.forward(x, residual)
        return out, l.backward(dout, kept)

    work(layer)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(layer)
    for k in range(3):
        x.copy_(inputs(64 + k, 192)[0][:64])
        graph.replay()
        layer.step()
        want = work(other)
        other.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        assert all(torch.equal(a, b) for a, b in zip(layer.grads + layer.params, other.grads + other.params)), k


@pytest.mark.parametrize("rows", [1, 5, 70])
@pytest.mark.parametrize("gated,norm", FORMS)
def test_answer_in_8_bits_follows_the_forward_pass(gated, norm, rows):
    layer = block(256, 512, gated=gated, norm=norm)
    x, residual, _ = inputs(rows, 256)
    out, _ = layer.forward(x, residual)
    got = layer.answer(x, residual, layer.eight_bits())
    # e4m3 is off by 2^-4 at most, 2^-5.3 in the mean, in both operands of a product whose terms are independent; three
    # such products in a gated layer
    near(got, R.f64(out), "answer", 2 * 2 ** 0.5 * 3 ** 0.5 * 2.0 ** -5.3)


def test_command():
    from paper_2606_16907_amd import measure_layer
    m = measure_layer.main(["--hidden", "256", "--ffn", "512", "--seq", "128", "--steps", "2", "--gated", "--norm", "layer", "--act", "silu"])
    assert m["rows"] == 128 and m["parameters"] == 3 * 256 * 512 + 3 * 256 + 2 * 512
    assert 0 < m["eta"] < 1 and abs(m["bytes_per_parameter"] - 16) < 1e-9
    assert m["plan_s_measured_eta"] > m["plan_s_eta_1"] > 0
    with pytest.raises(ValueError):
        measure_layer.FeedForward(8, 8, norm="batch")
