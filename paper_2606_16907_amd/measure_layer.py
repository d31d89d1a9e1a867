"""Measure a layer on this GPU, and plan with what was measured.

    python -m paper_2606_16907_amd.measure_layer [--hidden 1024] [--ffn 4096] [--seq 2048]
        [--micro-batch 1] [--act gelu] [--bits 32] [--steps 10] [--peak 2.5e15] [--instance tiny]

The plan search prices a layer's products at eta times an island's peak and its
parameters at 16 bytes each, and takes no time for the optimizer's step (the
profile() query of Tab. 2 is replaced by constants that the user brings).  This
runs the feed-forward half of a planned layer as it trains, with the operators
of `layer`: norm and residual, up projection with bias and activation, down
projection onto the residual stream, their gradients, and the AdamW step; and
prints the efficiency eta that its products reach, the optimizer's time and bytes
a parameter, and the plan of an instance with eta 1 and with the measured one.
The plan takes eta alone, as a part of the peak of every island's GPUs; attention
and gated projections are not among the operators and are taken to reach it too.
"""
from __future__ import annotations

import argparse
import copy
import json

import torch

from . import layer as L


class FeedForward:
    """norm -> up + activation -> down + residual, with its optimizer: bfloat16
    weights and gradients, float32 master copies, moments in 32 or 8 bits."""

    def __init__(self, hidden, ffn, act="gelu", bits=32, seed=0, eps=1e-6):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def weight(*shape, std):
            return torch.randn(shape, generator=gen, device="cuda") * std

        masters = [torch.ones(hidden, device="cuda"), weight(ffn, hidden, std=hidden ** -0.5),
                   torch.zeros(ffn, device="cuda"), weight(hidden, ffn, std=ffn ** -0.5),
                   torch.zeros(hidden, device="cuda")]
        params = [m.to(torch.bfloat16) for m in masters]
        self.norm, self.up, self.up_bias, self.down, self.down_bias = params
        self.params, self.masters = params, masters
        self.grads = [torch.zeros_like(p) for p in params]
        self.states = L.adamw_states(params, bits)
        scales = dict(m_scales=self.states[2], v_scales=self.states[3]) if bits == 8 else {}
        self.optimizer = L.AdamW(params, self.grads, self.states[0], self.states[1], masters=masters, **scales)
        self.act, self.eps, self.steps = act, eps, 0

    def forward(self, x, residual):
        """The residual stream behind the layer, and what backward() needs."""
        f = L.tg_rms_norm(x, self.norm, residual=residual, eps=self.eps)
        a, pre = L.tg_linear(f.y, self.up, bias=self.up_bias, act=self.act, keep_pre=True)
        out = L.tg_linear(a, self.down, bias=self.down_bias, residual=f.hidden)
        return out, (f, a, pre)

    def backward(self, dout, kept):
        """The gradient of x and residual; the weights' gradients go to their buffers."""
        f, a, pre = kept
        norm, up, up_bias, down, down_bias = self.grads
        da, _, _ = L.tg_linear_grad(dout, a, self.down, bias_grad=True, dw=down, dbias=down_bias)
        dy, _, _ = L.tg_linear_grad(da, f.y, self.up, pre=pre, act=self.act, bias_grad=True, dw=up, dbias=up_bias)
        dx, _ = L.tg_rms_norm_grad(dy, f.hidden, self.norm, f.rstd, dhidden=dout, dweight=norm)
        return dx

    def step(self, lr=1e-4, weight_decay=0.1):
        self.steps += 1
        self.optimizer.step(self.steps, lr, beta2=0.95, weight_decay=weight_decay, seed=self.steps)

    def eight_bits(self):
        """The up projection in 8 bits with a scale per output, for answer()."""
        scale = (self.up.float().abs().amax(1) / 448).clamp_min(1e-12)
        return (self.up.float() / scale[:, None]).to(L.E4M3), scale

    def answer(self, x, residual, up8):
        """forward() for a few new tokens: the norm's output and the up projection in 8 bits."""
        f = L.tg_rms_norm(x, self.norm, residual=residual, eps=self.eps, out_dtype=L.E4M3)
        a = L.tg_linear(f.y, up8[0], bias=self.up_bias, act=self.act, x_scale=f.scale, w_scale=up8[1])
        return L.tg_linear(a, self.down, bias=self.down_bias, residual=f.hidden)


def _seconds(work, steps):
    """Seconds of one call on the GPU, the median of `steps` after two untimed ones."""
    for _ in range(2):
        work()
    spans = []
    for _ in range(steps):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        work()
        end.record()
        spans.append((begin, end))
    torch.cuda.synchronize()
    return sorted(b.elapsed_time(e) for b, e in spans)[len(spans) // 2] / 1e3


def measure(hidden=1024, ffn=4096, seq=2048, micro_batch=1, act="gelu", bits=32, steps=10, peak=2.5e15):
    """Times of the feed-forward half of a layer on this GPU, and the efficiency its products reach."""
    layer = FeedForward(hidden, ffn, act, bits)
    rows = seq * micro_batch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x, residual, dout = (torch.randn((rows, hidden), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    dout *= 1e-2
    kept = layer.forward(x, residual)[1]
    up8 = layer.eight_bits()
    token = x[:1], residual[:1]
    forward = _seconds(lambda: layer.forward(x, residual), steps)
    backward = _seconds(lambda: layer.backward(dout, kept), steps)
    step = _seconds(layer.step, steps)
    answer = _seconds(lambda: layer.answer(*token, up8), steps)
    n = sum(p.numel() for p in layer.params)
    flops = 4.0 * rows * hidden * ffn  # forward, both projections; the gradients take twice that
    state = sum(t.numel() * t.element_size() for p in (layer.params, layer.grads, layer.masters, *layer.states) for t in p)
    return {"rows": rows, "parameters": n, "forward_s": forward, "backward_s": backward, "step_s": step, "one_token_s": answer,
            "eta": 3.0 * flops / (forward + backward) / peak, "step_ps_per_parameter": 1e12 * step / n,
            "bytes_per_parameter": state / n}


def plan(instance, eta):
    """The composed plan's iteration time for an instance whose islands reach `eta` of their peak."""
    from . import tangram as T
    inst = copy.deepcopy(instance)
    inst["space"]["eta"] = eta
    status, found, *_ = T.Problem(inst).plan_search()
    return found["T"] if status == T.TG_OK else None


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--ffn", type=int, default=4096)
    ap.add_argument("--seq", type=int, default=2048)
    ap.add_argument("--micro-batch", type=int, default=1)
    ap.add_argument("--act", choices=[a for a in L.ACTS if a], default="gelu")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32, help="of the optimizer's moments")
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--peak", type=float, default=2.5e15, help="FLOP/s that eta is a part of")
    ap.add_argument("--instance", default="tiny", help="instance to plan with eta 1 and the measured eta")
    a = ap.parse_args(argv)
    m = measure(a.hidden, a.ffn, a.seq, a.micro_batch, a.act, a.bits, a.steps, a.peak)
    from workloads import load_instance
    instance = load_instance(a.instance)
    m["instance"], m["plan_s_eta_1"], m["plan_s_measured_eta"] = a.instance, plan(instance, 1.0), plan(instance, m["eta"])
    print(json.dumps(m))
    return m


if __name__ == "__main__":
    main()
