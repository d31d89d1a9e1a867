"""Calls of the gated projections, the 8-bit product with a scale for each block of 128, its quantiser and the layer norm.

The plan search prices layers whose feed-forward half is gated (three matrices) or not (two).  These are the operators
that such a half runs on one GPU beside the plain matrix product, as it trains and as it answers with few tokens or in 8
bits.  Kinds (the field "op" of a case):
  gated       gate = x wg^T + bg and up = x wu^T + bu, y = act(gate) up, x [m, k], wg and wu [n, k]; in 8 bits x has a
              scale per row and each weight one per output.  With "grad" the pass is a training pass: y, gate and up as
              they are kept for it (in the inputs' type), then from dy the gradients of x, both weights and both biases
  block       y = act(x w^T + bias) + residual of 8-bit operands: x has a scale for every 128 consecutive values of a
              row, w one for every block of 128 x 128; scales are floats or powers of two (8 bits of exponent)
  quantise    values in 8 bits and their scales: of 128 consecutive values of a row, or of blocks of 128 x 128; the
              largest finite value of a block over its scale is at most 448
  layer_norm  h = x + residual, y = (h - mean) / sqrt(var + eps) * weight + bias, y in the inputs' type or in 8 bits with
              a scale per row.  With "grad" also, from h as it is kept, the gradients of x (which is the residual's too),
              of the weight and of the bias
`run` computes them with elementary torch operations in 32 bits where `own` is false, and with the library's entry points
where it is true.  `exact` has the floating-point results in 64 bits from the definitions.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
SCALES = {"f32": torch.float32, "powers": E8M0}
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -126
EPS = 1e-5
ACTS = ("none", "relu", "silu", "gelu")
BLOCK = 128  # values of a row (rows of a weight) that share a scale
MOST_FLOPS = 2.9e12


def _gated(name, m, k, n, type, act="silu", bias=False, grad=False, pad=0):
    return {"name": name, "op": "gated", "m": m, "k": k, "n": n, "type": type, "act": act, "bias": bias, "grad": grad,
            "pad": pad}


def _block(name, m, k, n, scales, act="none", bias=False, residual=False, pad=0):
    return {"name": name, "op": "block", "m": m, "k": k, "n": n, "scales": scales, "act": act, "bias": bias,
            "residual": residual, "pad": pad}


def _quantise(name, rows, cols, type, square, scales, pad=0):
    return {"name": name, "op": "quantise", "rows": rows, "cols": cols, "type": type, "square": square,
            "scales": scales, "pad": pad}


def _norm(name, rows, cols, type, out, residual=True, bias=True, grad=False, pad=0):
    return {"name": name, "op": "layer_norm", "rows": rows, "cols": cols, "type": type, "out": out,
            "residual": residual, "bias": bias, "grad": grad, "pad": pad}


def listed():
    return [
        # one new token through the 8B-like layer's gate and up projections: the latency of a weight-bound call
        _gated("gated_one_token", 1, 4096, 14336, "bf16"),
        # new tokens of a few dozen sequences, 8-bit weights: the 70B-like layer's on one of 8 tensor-parallel ranks
        _gated("gated_tokens_8bit", 48, 8192, 3584, "e4m3"),
        # sizes that fit no tile, rows that start at odd addresses: a padded batch cut down to its tokens, as it trains
        _gated("gated_ragged_step", 1531, 1001, 1367, "fp16", "gelu", bias=True, grad=True, pad=3),
        # a sequence of the 8B-like model as it trains: where the time of its step goes
        _gated("gated_step", 4096, 4096, 14336, "bf16", grad=True),
        # one new token through the 8B-like layer's down projection, onto the residual stream: the latency of a small call
        _block("block_one_token", 1, 14336, 4096, "f32", residual=True),
        # a long prompt through the 70B-like layer's down projection on a quarter of its columns
        _block("block_prompt", 8192, 7168, 8192, "f32", residual=True),
        # a batch of prompts whose tokens fill no tile, through the 8B-like layer's down projection
        _block("block_ragged_prompt", 5003, 14336, 4096, "powers"),
        # activations of a few new tokens in front of the down projection: the latency of a launch
        _quantise("quantise_tokens", 4, 14336, "bf16", False, "f32"),
        # a long prompt's activations in front of the 70B-like layer's down projection
        _quantise("quantise_prompt", 8192, 28672, "bf16", False, "powers"),
        # one new token each of four sequences of the largest model, quantised for an 8-bit product
        _norm("layer_norm_tokens_8bit", 4, 12288, "bf16", "e4m3"),
        # a micro-batch of the largest model, as it trains: the largest ordinary call
        _norm("layer_norm_step", 8192, 12288, "bf16", "same", grad=True),
        # rows of an odd length inside wider rows, in 32 bits
        _norm("layer_norm_ragged_step", 3001, 4999, "f32", "same", grad=True, pad=5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, whole):
    """A size of 16 times an odd number, rows of whole 16-byte units, or an odd one."""
    n = _log(rng, lo, hi)
    return n // 32 * 32 + 16 if whole else n | 1


def draw(rng):
    op = rng.choice(["gated", "gated", "gated", "block", "block", "quantise", "layer_norm", "layer_norm"])
    if op in ("gated", "block"):
        grad = op == "gated" and rng.random() < 0.5
        type = rng.choice(["bf16", "bf16", "fp16", "bf16" if grad else "e4m3"])
        # half of the calls serve few tokens or train one micro-batch; sizes of all kinds, odd ones among them
        m = _size(rng, 64, 8192, rng.random() < 0.5) if grad or rng.random() < 0.5 else _log(rng, 1, 64)
        whole = rng.random() < 0.6
        k, n = _size(rng, 256, 14336, whole), _size(rng, 256, 14336, whole)
        products = (6 if grad else 2) if op == "gated" else 1
        while 2.0 * m * k * n * products > MOST_FLOPS:
            m = m // 2 | 1
        case = {"op": op, "m": m, "k": k, "n": n, "act": rng.choice(ACTS), "bias": rng.random() < 0.5,
                "pad": rng.choice([0, 0, 16, 3])}
        if op == "gated":
            return {**case, "type": type, "grad": grad}
        return {**case, "scales": rng.choice(["f32", "powers"]), "residual": rng.random() < 0.5}
    type = rng.choice(["bf16", "bf16", "fp16", "f32"])
    if op == "quantise":
        cols = _size(rng, 64, 28672, rng.random() < 0.6)
        rows = _log(rng, 1, 64) if rng.random() < 0.3 else _size(rng, 64, max(64, min(16384, (1 << 27) // cols)), False)
        return {"op": op, "rows": rows, "cols": cols, "type": type, "square": rng.random() < 0.5,
                "scales": rng.choice(["f32", "powers"]), "pad": rng.choice([0, 0, 16, 5])}
    grad = rng.random() < 0.6
    cols = _size(rng, 64, 16384, rng.random() < 0.6)
    rows = _log(rng, 1, 64) if rng.random() < 0.3 else _size(rng, 64, max(64, min(16384, (1 << 26) // cols)), False)
    return {"op": op, "rows": rows, "cols": cols, "type": type, "out": "same" if grad or rng.random() < 0.4 else "e4m3",
            "residual": rng.random() < 0.7, "bias": rng.random() < 0.7, "grad": grad, "pad": rng.choice([0, 0, 16, 5])}


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _randn(gen, shape, dtype, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def _rows(gen, rows, cols, dtype, pad, std=1.0):
    """Rows of a buffer that is `pad` columns wider."""
    return _randn(gen, (rows, cols + pad), dtype, std)[:, :cols]


def _outliers(gen, rows, cols, dtype, pad):
    """Activations: columns of very different sizes, as behind a gated product."""
    size = torch.randn(cols + pad, generator=gen, device="cuda").mul_(1.5).exp_()
    return torch.randn((rows, cols + pad), generator=gen, device="cuda").mul_(size).to(dtype)[:, :cols]


def _quantised(t):
    """e4m3 values and a scale per row, as weights and activations are kept in 8 bits."""
    scale = (t.abs().amax(1) / E4M3_MAX).clamp_min(1e-12)
    return (t / scale[:, None]).to(E4M3), scale


def _wider(t, pad):
    """The same rows inside wider ones."""
    if pad == 0:
        return t
    out = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=torch.uint8, device="cuda").view(t.dtype)
    out[:, :t.shape[1]].copy_(t)
    return out[:, :t.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"gated": _prepare_gated, "block": _prepare_block, "quantise": _prepare_quantise,
            "layer_norm": _prepare_norm}[case["op"]](case, gen)


def _prepare_gated(case, gen):
    m, k, n, pad = case["m"], case["k"], case["n"], case["pad"]
    eight = case["type"] == "e4m3"
    dtype = torch.bfloat16 if eight else TYPES[case["type"]]
    s = {"case": case, "dtype": dtype, "x_scale": None, "wg_scale": None, "wu_scale": None, "dy": None}
    if eight:
        x, s["x_scale"] = _quantised(_randn(gen, (m, k), torch.float32))
        s["x"] = _wider(x, pad)
        s["wg"], s["wg_scale"] = _quantised(_randn(gen, (n, k), torch.float32, k ** -0.5))
        s["wu"], s["wu_scale"] = _quantised(_randn(gen, (n, k), torch.float32, k ** -0.5))
    else:
        s["x"] = _rows(gen, m, k, dtype, pad)
        s["wg"], s["wu"] = (_randn(gen, (n, k), dtype, k ** -0.5) for _ in range(2))
    s["bg"], s["bu"] = (_randn(gen, (n,), dtype, 0.1) if case["bias"] else None for _ in range(2))
    if case["grad"]:
        s["dy"] = _rows(gen, m, n, dtype, pad, 0.05)
    return s


def _prepare_block(case, gen):
    m, k, n, pad = case["m"], case["k"], case["n"], case["pad"]
    s = {"case": case}
    x, s["x_scale"] = _to_blocks(_outliers(gen, m, k, torch.float32, 0), False, case["scales"])
    w, s["w_scale"] = _to_blocks(_randn(gen, (n, k), torch.float32, k ** -0.5), True, case["scales"])
    s["x"], s["w"] = _wider(x, pad), _wider(w, pad)
    s["bias"] = _randn(gen, (n,), torch.bfloat16, 0.1) if case["bias"] else None
    s["residual"] = _rows(gen, m, n, torch.bfloat16, pad) if case["residual"] else None
    return s


def _prepare_quantise(case, gen):
    return {"case": case, "x": _outliers(gen, case["rows"], case["cols"], TYPES[case["type"]], case["pad"])}


def _prepare_norm(case, gen):
    rows, cols, pad, dtype = case["rows"], case["cols"], case["pad"], TYPES[case["type"]]
    s = {"case": case, "x": _rows(gen, rows, cols, dtype, pad), "dy": None, "dh": None,
         "weight": (1.0 + _randn(gen, (cols,), torch.float32, 0.1)).to(dtype),
         "bias": _randn(gen, (cols,), dtype, 0.1) if case["bias"] else None,
         "residual": (_rows(gen, rows, cols, torch.float32, pad, 2.0) + 0.5).to(dtype) if case["residual"] else None}
    if case["grad"]:
        s["dy"] = _rows(gen, rows, cols, dtype, pad, 0.05)
        s["dh"] = _rows(gen, rows, cols, dtype, pad, 0.05) if case["residual"] else None
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return {"gated": _own_gated, "block": _own_block, "quantise": _own_quantise, "layer_norm": _own_norm}[op](s)
    return {"gated": _plain_gated, "block": _plain_block, "quantise": _plain_quantise, "layer_norm": _plain_norm}[op](s)


def _own_gated(s):
    from paper_2606_16907_amd import layer
    c = s["case"]
    if not c["grad"]:
        return layer.tg_gated(s["x"], s["wg"], s["wu"], gate_bias=s["bg"], up_bias=s["bu"], act=c["act"],
                              x_scale=s["x_scale"], gate_scale=s["wg_scale"], up_scale=s["wu_scale"], out_dtype=s["dtype"])
    y, gate, up = layer.tg_gated(s["x"], s["wg"], s["wu"], gate_bias=s["bg"], up_bias=s["bu"], act=c["act"], keep_pre=True)
    g = layer.tg_gated_grad(s["dy"], s["x"], s["wg"], s["wu"], gate, up, act=c["act"], bias_grad=c["bias"])
    return {"y": y, "gate": gate, "up": up, "dx": g.dx, "dwg": g.dw_gate, "dwu": g.dw_up, "dbg": g.dgate_bias,
            "dbu": g.dup_bias}


def _own_block(s):
    from paper_2606_16907_amd import layer
    return layer.tg_block_linear(s["x"], s["w"], s["x_scale"], s["w_scale"], bias=s["bias"], act=s["case"]["act"],
                                 residual=s["residual"], out_dtype=torch.bfloat16)


def _own_quantise(s):
    from paper_2606_16907_amd import layer
    c = s["case"]
    q = layer.tg_quantize(s["x"], block_rows=BLOCK if c["square"] else 1, scale_dtype=SCALES[c["scales"]])
    return {"y": q.y, "scale": q.scale}


def _own_norm(s):
    from paper_2606_16907_amd import layer
    c = s["case"]
    f = layer.tg_layer_norm(s["x"], s["weight"], bias=s["bias"], residual=s["residual"], eps=EPS,
                            out_dtype=E4M3 if c["out"] == "e4m3" else s["x"].dtype)
    out = {"y": f.y, "scale": f.scale, "hidden": f.hidden if c["residual"] else None}
    if c["grad"]:
        out["dx"], out["dweight"], out["dbias"] = layer.tg_layer_norm_grad(
            s["dy"], f.hidden, s["weight"], f.mean, f.rstd, dhidden=s["dh"], bias_grad=c["bias"])
    return out


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        t = 1 / (1 + torch.exp(-z))
        return t * (1 + z * (1 - t))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _plain_gated(s):
    c, dtype = s["case"], s["dtype"]
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    gate, up = x @ wg.t(), x @ wu.t()
    if s["x_scale"] is not None:
        gate, up = gate * s["x_scale"][:, None] * s["wg_scale"], up * s["x_scale"][:, None] * s["wu_scale"]
    if c["bias"]:
        gate, up = gate + s["bg"].float(), up + s["bu"].float()
    y = (_act(gate, c["act"]) * up).to(dtype)
    if not c["grad"]:
        return y
    # the gradient reads gate and up as the forward pass keeps them
    kept_gate, kept_up = gate.to(dtype), up.to(dtype)
    dy, gate, up = s["dy"].float(), kept_gate.float(), kept_up.float()
    dg, du = dy * up * _act_grad(gate, c["act"]), dy * _act(gate, c["act"])
    return {"y": y, "gate": kept_gate, "up": kept_up, "dx": (dg @ wg + du @ wu).to(dtype), "dwg": (dg.t() @ x).to(dtype),
            "dwu": (du.t() @ x).to(dtype), "dbg": dg.sum(0).to(dtype) if c["bias"] else None,
            "dbu": du.sum(0).to(dtype) if c["bias"] else None}


def _spread(scale, rows, cols, square):
    """A block's scale at each of its values."""
    t = scale.float().repeat_interleave(BLOCK, 1)[:, :cols]
    return t.repeat_interleave(BLOCK, 0)[:rows] if square else t


def _to_blocks(x, square, scales):
    """e4m3 values of x and the scales of their blocks."""
    rows, cols = x.shape
    nr, nc = -(-rows // BLOCK) if square else rows, -(-cols // BLOCK)
    a = x.float().abs()
    a = torch.where(a < math.inf, a, torch.zeros_like(a))
    a = torch.nn.functional.pad(a, (0, nc * BLOCK - cols, 0, nr * BLOCK - rows if square else 0))
    most = a.view(nr, BLOCK, nc, BLOCK).amax((1, 3)) if square else a.view(nr, nc, BLOCK).amax(2)
    scale = (most / E4M3_MAX).clamp_min(LEAST_SCALE)
    if scales == "powers":  # the least power of two that is no smaller
        part, exponent = torch.frexp(scale)
        scale = torch.ldexp(torch.ones_like(part), torch.where(part == 0.5, exponent - 1, exponent))
    scale = torch.where(most > 0, scale, torch.ones_like(scale))
    q = (x.float() / _spread(scale, rows, cols, square)).to(E4M3)
    return q, scale.to(SCALES[scales])


def _plain_block(s):
    c = s["case"]
    m, k, n = c["m"], c["k"], c["n"]
    z = (s["x"].float() * _spread(s["x_scale"], m, k, False)) @ (s["w"].float() * _spread(s["w_scale"], n, k, True)).t()
    if c["bias"]:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if c["residual"]:
        y = y + s["residual"].float()
    return y.to(torch.bfloat16)


def _plain_quantise(s):
    c = s["case"]
    q, scale = _to_blocks(s["x"], c["square"], c["scales"])
    return {"y": q, "scale": scale}


def _plain_norm(s):
    c, dtype = s["case"], s["x"].dtype
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    mean = h.mean(1, keepdim=True)
    centred = h - mean
    rstd = 1 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
    w = s["weight"].float()
    y = centred * rstd * w
    if c["bias"]:
        y = y + s["bias"].float()
    out = {"y": y.to(dtype), "scale": None, "hidden": h.to(dtype) if c["residual"] else None}
    if c["out"] == "e4m3":
        scale = (y.abs().amax(1) / E4M3_MAX).clamp_min(LEAST_SCALE)
        out["y"], out["scale"] = (y / scale[:, None]).to(E4M3), scale
    if c["grad"]:
        dy = s["dy"].float()
        xhat = (h.to(dtype).float() - mean) * rstd
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        out["dx"] = (dx + s["dh"].float() if s["dh"] is not None else dx).to(dtype)
        out["dweight"] = (dy * xhat).sum(0).to(dtype)
        out["dbias"] = dy.sum(0).to(dtype) if c["bias"] else None
    return out


# ----------------------------------------------------------------------------
# work and 64-bit results
# ----------------------------------------------------------------------------
def work(case):
    if case["op"] == "gated":
        m, k, n = case["m"], case["k"], case["n"]
        e, b = 1 if case["type"] == "e4m3" else 2, 2 * n * case["bias"]
        nbytes = e * (m * k + 2 * n * k) + 2 * m * n + 2 * b
        nbytes += 4 * (m + 2 * n) if case["type"] == "e4m3" else 0
        flops = 4.0 * m * k * n
        if case["grad"]:  # gate and up kept, dy read, dx and both weights' gradients written, the biases' gradients
            nbytes += 2 * (2 * m * n + m * n + m * k + 2 * n * k) + 2 * b
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "block":
        m, k, n = case["m"], case["k"], case["n"]
        kb, e = -(-k // BLOCK), 4 if case["scales"] == "f32" else 1
        nbytes = m * k + n * k + e * kb * (m + -(-n // BLOCK)) + 2 * m * n * (1 + case["residual"]) + 2 * n * case["bias"]
        return {"bytes": nbytes, "flops": 2.0 * m * k * n}
    rows, cols, e = case["rows"], case["cols"], 4 if case["type"] == "f32" else 2
    n = rows * cols
    if case["op"] == "quantise":
        blocks = (-(-rows // BLOCK) if case["square"] else rows) * -(-cols // BLOCK)
        return {"bytes": (e + 1) * n + (4 if case["scales"] == "f32" else 1) * blocks, "flops": 3.0 * n}
    nbytes = e * n * (1 + 2 * case["residual"]) + e * cols * (1 + case["bias"])
    nbytes += n + 4 * rows if case["out"] == "e4m3" else e * n
    flops = 8.0 * n
    if case["grad"]:  # dy and the residual stream's gradient read, dx and the gradients of weight and bias written
        nbytes += e * n * (2 + case["residual"]) + e * cols * (1 + case["bias"])
        flops += 12.0 * n
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _exact_gated, "block": _exact_block, "quantise": _exact_quantise,
            "layer_norm": _exact_norm}[case["op"]](s)


def _exact_slope(z, act):
    """(act(z), its slope) in 64 bits."""
    zero = torch.zeros((), dtype=z.dtype, device="cuda")
    if act == "relu":
        return torch.maximum(z, zero), torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    if act == "silu":
        t = torch.sigmoid(z)
        return z * t, t + z * t * (1 - t)
    if act == "gelu":
        normal = torch.distributions.Normal(zero, zero + 1)
        return z * normal.cdf(z), normal.cdf(z) + z * torch.exp(normal.log_prob(z))
    return z, torch.ones_like(z)


def _exact_gated(s):
    c, f64 = s["case"], torch.float64
    x, wg, wu = (s[key].to(f64) for key in ("x", "wg", "wu"))
    if s["x_scale"] is not None:
        x = x * s["x_scale"].to(f64)[:, None]
        wg, wu = wg * s["wg_scale"].to(f64)[:, None], wu * s["wu_scale"].to(f64)[:, None]
    gate, up = torch.mm(x, wg.t().contiguous()), torch.mm(x, wu.t().contiguous())
    if c["bias"]:
        gate, up = gate + s["bg"].to(f64), up + s["bu"].to(f64)
    y = _exact_slope(gate, c["act"])[0] * up
    if not c["grad"]:
        return y
    kept_gate, kept_up = gate.to(s["dtype"]).to(f64), up.to(s["dtype"]).to(f64)
    value, slope = _exact_slope(kept_gate, c["act"])
    dy = s["dy"].to(f64)
    dg, du = dy * kept_up * slope, dy * value
    return {"y": y, "gate": gate, "up": up, "dx": torch.mm(dg, wg) + torch.mm(du, wu),
            "dwg": torch.mm(dg.t().contiguous(), x), "dwu": torch.mm(du.t().contiguous(), x),
            "dbg": dg.sum(0) if c["bias"] else None, "dbu": du.sum(0) if c["bias"] else None}


def _exact_values(q, scale, square):
    """What 8-bit values stand for, in 64 bits."""
    at = [torch.arange(n, device="cuda") // BLOCK for n in q.shape]
    t = scale.float().to(torch.float64)[:, at[1]]
    return q.to(torch.float64) * (t[at[0]] if square else t)


def _exact_block(s):
    c, f64 = s["case"], torch.float64
    x, w = _exact_values(s["x"], s["x_scale"], False), _exact_values(s["w"], s["w_scale"], True)
    z = torch.mm(x, w.t().contiguous())
    if c["bias"]:
        z += s["bias"].to(f64)
    y = _exact_slope(z, c["act"])[0]
    return y + s["residual"].to(f64) if c["residual"] else y


def _exact_quantise(s):
    c = s["case"]
    x = s["x"].to(torch.float64)
    rows, cols = x.shape
    at_row = torch.arange(rows, device="cuda") // (BLOCK if c["square"] else 1)
    at_col = torch.arange(cols, device="cuda") // BLOCK
    size = (int(at_row[-1]) + 1, int(at_col[-1]) + 1)
    place = (at_row[:, None] * size[1] + at_col).reshape(-1)
    most = torch.zeros(size[0] * size[1], dtype=torch.float64, device="cuda")
    most.scatter_reduce_(0, place, x.abs().reshape(-1), "amax")
    scale = (most / E4M3_MAX).clamp_min(LEAST_SCALE)
    if c["scales"] == "powers":
        scale = torch.exp2(torch.ceil(torch.log2(scale)))
    scale = torch.where(most > 0, scale, torch.ones_like(scale))
    return {"y": x / scale[place].view(rows, cols), "scale": scale.view(size)}


def _exact_norm(s):
    c, f64 = s["case"], torch.float64
    h = s["x"].to(f64)
    if s["residual"] is not None:
        h = h + s["residual"].to(f64)
    cols = h.shape[1]
    mean = h.sum(1, keepdim=True) / cols
    root = ((h - mean).square().sum(1, keepdim=True) / cols + EPS).sqrt()
    w = s["weight"].to(f64)
    y = (h - mean) / root * w
    if c["bias"]:
        y = y + s["bias"].to(f64)
    out = {"y": y, "scale": None, "hidden": h if c["residual"] else None}
    if c["out"] == "e4m3":
        out["scale"] = y.abs().amax(1) / E4M3_MAX
        out["y"] = y / out["scale"][:, None]
    if c["grad"]:
        dy = s["dy"].to(f64)
        xhat = (h.to(s["x"].dtype).to(f64) - mean) / root
        g = dy * w
        dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) / root
        out["dx"] = dx if s["dh"] is None else dx + s["dh"].to(f64)
        out["dweight"] = (dy * xhat).sum(0)
        out["dbias"] = dy.sum(0) if c["bias"] else None
    return out
