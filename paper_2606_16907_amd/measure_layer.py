"""Measure a layer on this GPU, and plan with what was measured.

    python -m paper_2606_16907_amd.measure_layer [--hidden 1024] [--ffn 4096] [--seq 2048]
        [--micro-batch 1] [--act gelu] [--gated] [--norm rms] [--bits 32] [--steps 10] [--peak 2.5e15]
        [--instance tiny]

The plan search prices a layer's products at eta times an island's peak and its
parameters at 16 bytes each, and takes no time for the optimizer's step (the
profile() query of Tab. 2 is replaced by constants that the user brings).  This
runs the feed-forward half of a planned layer as it trains, with the operators
of `layer`: norm and residual, up projection with bias and activation (or gate and
up projections, the activation and their product), down projection onto the
residual stream, their gradients, and the AdamW step; and a token in 8 bits.  It
prints the efficiency eta that its products reach, the optimizer's time and bytes
a parameter, and the plan of an instance with eta 1 and with the measured one.
The plan takes eta alone, as a part of the peak of every island's GPUs; attention
is not among the operators and is taken to reach it too.
"""
from __future__ import annotations

import argparse
import copy
import json

import torch

from . import layer as L


class FeedForward:
    """norm -> up + activation -> down + residual, with its optimizer: bfloat16
    weights and gradients, float32 master copies, moments in 32 or 8 bits.
    gated: act(gate) up in the place of act(up).  norm: "rms" or "layer"."""

    def __init__(self, hidden, ffn, act="gelu", bits=32, seed=0, eps=1e-6, gated=False, norm="rms"):
        if norm not in ("rms", "layer"):
            raise ValueError(f"norm: {norm!r}, rms or layer expected")
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def weight(*shape, std):
            return torch.randn(shape, generator=gen, device="cuda") * std

        masters = {"norm": torch.ones(hidden, device="cuda"), "up": weight(ffn, hidden, std=hidden ** -0.5),
                   "up_bias": torch.zeros(ffn, device="cuda"), "down": weight(hidden, ffn, std=ffn ** -0.5),
                   "down_bias": torch.zeros(hidden, device="cuda")}
        if gated:
            masters["gate"] = weight(ffn, hidden, std=hidden ** -0.5)
            masters["gate_bias"] = torch.zeros(ffn, device="cuda")
        if norm == "layer":
            masters["norm_bias"] = torch.zeros(hidden, device="cuda")
        self.masters = list(masters.values())
        self.params = [m.to(torch.bfloat16) for m in self.masters]
        self.grads = [torch.zeros_like(p) for p in self.params]
        for name, param in zip(masters, self.params):
            setattr(self, name, param)
        self.grad = dict(zip(masters, self.grads))
        self.states = L.adamw_states(self.params, bits)
        scales = dict(m_scales=self.states[2], v_scales=self.states[3]) if bits == 8 else {}
        self.optimizer = L.AdamW(self.params, self.grads, self.states[0], self.states[1], masters=self.masters, **scales)
        self.act, self.eps, self.steps, self.gated, self.layer_norm = act, eps, 0, gated, norm == "layer"

    def normed(self, x, residual, out_dtype=None):
        if self.layer_norm:
            return L.tg_layer_norm(x, self.norm, bias=self.norm_bias, residual=residual, eps=self.eps, out_dtype=out_dtype)
        return L.tg_rms_norm(x, self.norm, residual=residual, eps=self.eps, out_dtype=out_dtype)

    def forward(self, x, residual):
        """The residual stream behind the layer, and what backward() needs."""
        f = self.normed(x, residual)
        if self.gated:
            a, gate, up = L.tg_gated(f.y, self.gate, self.up, gate_bias=self.gate_bias, up_bias=self.up_bias, act=self.act,
                                     keep_pre=True)
            pre = gate, up
        else:
            a, pre = L.tg_linear(f.y, self.up, bias=self.up_bias, act=self.act, keep_pre=True)
        out = L.tg_linear(a, self.down, bias=self.down_bias, residual=f.hidden)
        return out, (f, a, pre)

    def backward(self, dout, kept):
        """The gradient of x and residual; the weights' gradients go to their buffers."""
        f, a, pre = kept
        g = self.grad
        da, _, _ = L.tg_linear_grad(dout, a, self.down, bias_grad=True, dw=g["down"], dbias=g["down_bias"])
        if self.gated:
            dy = L.tg_gated_grad(da, f.y, self.gate, self.up, *pre, act=self.act, bias_grad=True, dw_gate=g["gate"],
                                 dw_up=g["up"], dgate_bias=g["gate_bias"], dup_bias=g["up_bias"]).dx
        else:
            dy, _, _ = L.tg_linear_grad(da, f.y, self.up, pre=pre, act=self.act, bias_grad=True, dw=g["up"],
                                        dbias=g["up_bias"])
        if self.layer_norm:
            return L.tg_layer_norm_grad(dy, f.hidden, self.norm, f.mean, f.rstd, dhidden=dout, dweight=g["norm"],
                                        dbias=g["norm_bias"])[0]
        return L.tg_rms_norm_grad(dy, f.hidden, self.norm, f.rstd, dhidden=dout, dweight=g["norm"])[0]

    def step(self, lr=1e-4, weight_decay=0.1):
        self.steps += 1
        self.optimizer.step(self.steps, lr, beta2=0.95, weight_decay=weight_decay, seed=self.steps)

    def eight_bits(self):
        """What answer() takes: the up projection in 8 bits with a scale per output; of a gated layer the gate and up
        projections so, and the down projection with a scale for every block of 128 x 128."""
        def rows(w):
            scale = (w.float().abs().amax(1) / 448).clamp_min(1e-12)
            return (w.float() / scale[:, None]).to(L.E4M3), scale
        if self.gated:
            return rows(self.gate), rows(self.up), L.tg_quantize(self.down, block_rows=L.BLOCK)
        return rows(self.up)

    def answer(self, x, residual, eight):
        """forward() for a few new tokens in 8 bits: the norm's output and the up projection, and of a gated layer the
        gate and down projections too."""
        f = self.normed(x, residual, L.E4M3)
        if self.gated:
            (gate, gate_scale), (up, up_scale), down = eight
            a = L.tg_gated(f.y, gate, up, gate_bias=self.gate_bias, up_bias=self.up_bias, act=self.act, x_scale=f.scale,
                           gate_scale=gate_scale, up_scale=up_scale)
            q = L.tg_quantize(a)
            return L.tg_block_linear(q.y, down.y, q.scale, down.scale, bias=self.down_bias, residual=f.hidden)
        a = L.tg_linear(f.y, eight[0], bias=self.up_bias, act=self.act, x_scale=f.scale, w_scale=eight[1])
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


def measure(hidden=1024, ffn=4096, seq=2048, micro_batch=1, act="gelu", bits=32, steps=10, peak=2.5e15, gated=False,
            norm="rms"):
    """Times of the feed-forward half of a layer on this GPU, and the efficiency its products reach."""
    layer = FeedForward(hidden, ffn, act, bits, gated=gated, norm=norm)
    rows = seq * micro_batch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x, residual, dout = (torch.randn((rows, hidden), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    dout *= 1e-2
    kept = layer.forward(x, residual)[1]
    eight = layer.eight_bits()
    token = x[:1], residual[:1]
    forward = _seconds(lambda: layer.forward(x, residual), steps)
    backward = _seconds(lambda: layer.backward(dout, kept), steps)
    step = _seconds(layer.step, steps)
    answer = _seconds(lambda: layer.answer(*token, eight), steps)
    n = sum(p.numel() for p in layer.params)
    flops = 2.0 * (3 if gated else 2) * rows * hidden * ffn  # forward, the projections; the gradients take twice that
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
    ap.add_argument("--gated", action="store_true", help="gate and up projections")
    ap.add_argument("--norm", choices=("rms", "layer"), default="rms")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32, help="of the optimizer's moments")
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--peak", type=float, default=2.5e15, help="FLOP/s that eta is a part of")
    ap.add_argument("--instance", default="tiny", help="instance to plan with eta 1 and the measured eta")
    a = ap.parse_args(argv)
    m = measure(a.hidden, a.ffn, a.seq, a.micro_batch, a.act, a.bits, a.steps, a.peak, a.gated, a.norm)
    from workloads import load_instance
    instance = load_instance(a.instance)
    m["instance"], m["plan_s_eta_1"], m["plan_s_measured_eta"] = a.instance, plan(instance, 1.0), plan(instance, m["eta"])
    print(json.dumps(m))
    return m


if __name__ == "__main__":
    main()
