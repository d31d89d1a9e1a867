"""Calls of the layer operators, for timing: what one planned layer runs on one GPU of an island.

The plan search prices a layer by its matrix products and its parameters; these
are the operators behind those prices, as they are called when the layer trains
(forward, backward, optimizer step) and when it answers with few tokens or in
8 bits.  Kinds (the field "op" of a case):
  linear    y = act(x w^T + bias) + residual, x [m, k], w [n, k]; in 8 bits x
            has a scale per row and w one per output.  With "grad" the pass is a
            training pass: y, then from dy the gradients of x, w and bias
  rms_norm  h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, y in the
            inputs' type or in 8 bits with a scale per row.  With "grad" also
            the gradients of x (which is the residual's too) and of the weight
  adamw     one step over all tensors of some layers, 16-bit weights with
            32-bit master copies, moments in 32 bits or in 8 with a scale per
            256 values, rounded with given random bits (a hash of the seed, the
            tensor and the element)
`run` computes them with elementary torch operations in 32 bits where `own` is
false, and with the library's entry points where it is true.  `exact` has the
floating-point results in 64 bits from the definitions.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
EPS = 1e-6
ACTS = ("none", "relu", "silu", "gelu")
BLOCK = 256  # values of an 8-bit state that share a scale
LR, BETA1, BETA2, ADAM_EPS, DECAY = 5e-5, 0.9, 0.95, 1e-8, 0.1
MOST_FLOPS, MOST_BYTES = 3.7e12, 7.0e9


def _linear(name, m, k, n, type, act="none", bias=False, residual=False, grad=False, pad=0):
    return {"name": name, "op": "linear", "m": m, "k": k, "n": n, "type": type, "act": act, "bias": bias,
            "residual": residual, "grad": grad, "pad": pad}


def _norm(name, rows, cols, type, out, residual=True, grad=False, pad=0):
    return {"name": name, "op": "rms_norm", "rows": rows, "cols": cols, "type": type, "out": out,
            "residual": residual, "grad": grad, "pad": pad}


def _adamw(name, layers, hidden, kv, ffn, mats, bits):
    return {"name": name, "op": "adamw", "layers": layers, "hidden": hidden, "kv": kv, "ffn": ffn, "mats": mats,
            "bits": bits}


def listed():
    return [
        # one new token through the up projection of the 8B-like layer: the latency of a weight-bound call
        _linear("linear_one_token", 1, 4096, 14336, "bf16", "gelu", bias=True),
        # a few dozen sequences' new tokens, 8-bit weights: the 70B-like layer's FFN on a quarter of its columns
        _linear("linear_tokens_8bit", 48, 8192, 7168, "e4m3"),
        # a micro-batch of one sequence through the small model's up projection, as it trains
        _linear("linear_small_step", 2048, 1024, 4096, "bf16", "gelu", bias=True, grad=True),
        # sizes that fit no tile, rows that start at odd addresses: a padded batch cut down to its tokens
        _linear("linear_ragged_step", 1531, 1001, 2047, "fp16", "relu", bias=True, residual=True, grad=True, pad=3),
        # the largest model's up projection on one of 8 tensor-parallel ranks, as it trains: where the time of a step goes
        _linear("linear_large_step", 8192, 12288, 6144, "bf16", "gelu", bias=True, grad=True),
        # a long prompt through the 70B-like layer's down projection in 8 bits, onto the residual stream
        _linear("linear_8bit_prompt", 8192, 7168, 8192, "e4m3", residual=True),
        # one new token each of four sequences, quantised for the 8-bit product: the latency of a small call
        _norm("norm_tokens_8bit", 4, 8192, "bf16", "e4m3"),
        # a micro-batch of the 70B-like layer, as it trains: the largest ordinary call
        _norm("norm_step", 8192, 8192, "bf16", "same", grad=True),
        # rows of an odd length inside wider rows, in 32 bits
        _norm("norm_ragged_step", 3001, 4999, "f32", "same", grad=True, pad=5),
        # the shard of a small layer: many short tensors, bound by the launch
        _adamw("adamw_short_tensors", 4, 97, 97, 389, 2, 32),
        # all eight layers of the small model, states in 32 bits
        _adamw("adamw_small_model", 8, 1024, 1024, 4096, 2, 32),
        # two layers of the 8B-like model on one rank, states in 8 bits: the largest step
        _adamw("adamw_8bit", 2, 4096, 1024, 14336, 3, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, whole):
    """A size of 16 times an odd number, rows of whole 16-byte units, or an odd one."""
    n = _log(rng, lo, hi)
    return n // 32 * 32 + 16 if whole else n | 1


def draw(rng):
    op = rng.choice(["linear", "linear", "rms_norm", "adamw"])
    if op == "linear":
        type = rng.choice(["bf16", "bf16", "fp16", "e4m3"])
        grad = type != "e4m3" and rng.random() < 0.5
        # half of the calls serve few tokens or train one micro-batch; sizes of all kinds, odd ones among them
        m = _size(rng, 64, 8192, rng.random() < 0.5) if grad or rng.random() < 0.5 else _log(rng, 1, 64)
        whole = type == "e4m3" or rng.random() < 0.6
        k, n = _size(rng, 256, 14336, whole), _size(rng, 256, 14336, whole)
        passes = 3 if grad else 1
        while 2.0 * m * k * n * passes > MOST_FLOPS:
            m = m // 2 | 1
        return {"op": op, "m": m, "k": k, "n": n, "type": type, "act": rng.choice(ACTS), "bias": rng.random() < 0.5,
                "residual": rng.random() < 0.5, "grad": grad, "pad": rng.choice([0, 0, 16, 3]) if type != "e4m3" else 0}
    if op == "rms_norm":
        type = rng.choice(["bf16", "bf16", "fp16", "f32"])
        grad = rng.random() < 0.6
        cols = _size(rng, 64, 16384, rng.random() < 0.6)
        rows = _log(rng, 1, 64) if rng.random() < 0.3 else _size(rng, 64, max(64, min(16384, (1 << 26) // cols)), False)
        return {"op": op, "rows": rows, "cols": cols, "type": type, "out": "same" if grad or rng.random() < 0.4 else "e4m3",
                "residual": rng.random() < 0.7, "grad": grad, "pad": rng.choice([0, 0, 16, 5])}
    while True:
        whole = rng.random() < 0.6
        hidden = _size(rng, 64, 4096, whole)
        case = {"op": op, "layers": rng.randint(1, 8), "hidden": hidden, "kv": hidden // rng.choice([1, 4, 8]),
                "ffn": _size(rng, 2 * hidden, 4 * hidden, whole), "mats": rng.choice([2, 3]), "bits": rng.choice([8, 32])}
        if work(case)["bytes"] <= MOST_BYTES:
            return case


def _tensor_sizes(case):
    """Parameters of each tensor: attention's four matrices, the FFN's two or three, two norms, layer by layer."""
    h, kv, f = case["hidden"], case["kv"], case["ffn"]
    return ([h * h, h * kv, h * kv, h * h] + [h * f] * case["mats"] + [h, h]) * case["layers"]


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _randn(gen, shape, dtype, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def _rows(gen, rows, cols, dtype, pad, std=1.0):
    """Rows of a buffer that is `pad` columns wider."""
    return _randn(gen, (rows, cols + pad), dtype, std)[:, :cols]


def _quantised(t):
    """e4m3 values and a scale per row, as weights and activations are kept in 8 bits."""
    scale = (t.abs().amax(1) / E4M3_MAX).clamp_min(1e-12)
    return (t / scale[:, None]).to(E4M3), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"linear": _prepare_linear, "rms_norm": _prepare_norm, "adamw": _prepare_adamw}[case["op"]](case, gen, seed)


def _prepare_linear(case, gen, seed):
    m, k, n, pad = case["m"], case["k"], case["n"], case["pad"]
    eight = case["type"] == "e4m3"
    dtype = torch.bfloat16 if eight else TYPES[case["type"]]
    s = {"case": case, "dtype": dtype, "x_scale": None, "w_scale": None, "dy": None}
    if eight:
        s["x"], s["x_scale"] = _quantised(_randn(gen, (m, k), torch.float32))
        s["w"], s["w_scale"] = _quantised(_randn(gen, (n, k), torch.float32, k ** -0.5))
    else:
        s["x"] = _rows(gen, m, k, dtype, pad)
        s["w"] = _randn(gen, (n, k), dtype, k ** -0.5)
    s["bias"] = _randn(gen, (n,), dtype, 0.1) if case["bias"] else None
    s["residual"] = _rows(gen, m, n, dtype, pad) if case["residual"] else None
    if case["grad"]:
        s["dy"] = _rows(gen, m, n, dtype, pad, 0.05)
    return s


def _prepare_norm(case, gen, seed):
    rows, cols, pad, dtype = case["rows"], case["cols"], case["pad"], TYPES[case["type"]]
    s = {"case": case, "x": _rows(gen, rows, cols, dtype, pad), "dy": None, "dh": None,
         "weight": (1.0 + _randn(gen, (cols,), torch.float32, 0.1)).to(dtype),
         "residual": _rows(gen, rows, cols, dtype, pad, 2.0) if case["residual"] else None}
    if case["grad"]:
        s["dy"] = _rows(gen, rows, cols, dtype, pad, 0.05)
        s["dh"] = _rows(gen, rows, cols, dtype, pad, 0.05) if case["residual"] else None
    return s


def _prepare_adamw(case, gen, seed):
    sizes = _tensor_sizes(case)
    blocks = [-(-n // BLOCK) for n in sizes]
    total = sum(blocks) * BLOCK
    s = {"case": case, "seed": seed & 0x7FFFFFFF, "step": 1000, "opt": None}
    # one flat buffer a kind, a tensor begins at a whole block; what lies between the tensors is zero and stays zero
    per = torch.tensor(blocks, device="cuda")
    first = per.cumsum(0) - per
    s["tensor"] = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), per)
    s["block"] = torch.arange(sum(blocks), device="cuda") - first[s["tensor"]]
    live = (s["block"][:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
            < torch.tensor(sizes, device="cuda")[s["tensor"]][:, None]).reshape(-1)
    s["master"] = _randn(gen, total, torch.float32, 0.02).mul_(live)
    s["param"] = s["master"].to(torch.bfloat16)
    s["grad"] = _randn(gen, total, torch.bfloat16, 1e-3).mul_(live)
    m = _randn(gen, total, torch.float32, 3e-4).mul_(live)
    r = torch.rand(total, generator=gen, device="cuda").add_(0.5).mul_(1e-3).mul_(live)
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _quantised(m.view(-1, BLOCK))
        s["v"], s["v_scale"] = _quantised(r.view(-1, BLOCK))
        s["m"], s["v"] = s["m"].view(-1), s["v"].view(-1)
    else:
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, r.square_(), None, None
    if own:  # the plan over the tensors, kept as long as they are
        from paper_2606_16907_amd import layer
        at = [int(b) * BLOCK for b in first.tolist()]
        parts = lambda t: [t[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
        scales = lambda t: None if t is None else [t[a // BLOCK:a // BLOCK + b] for a, b in zip(at, blocks)]  # noqa: E731
        s["opt"] = layer.AdamW(parts(s["param"]), parts(s["grad"]), parts(s["m"]), parts(s["v"]),
                               m_scales=scales(s["m_scale"]), v_scales=scales(s["v_scale"]), masters=parts(s["master"]))
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return {"linear": _own_linear, "rms_norm": _own_norm, "adamw": _own_adamw}[op](s)
    return {"linear": _plain_linear, "rms_norm": _plain_norm, "adamw": _plain_adamw}[op](s)


def _own_linear(s):
    from paper_2606_16907_amd import layer
    c = s["case"]
    if not c["grad"]:
        return layer.tg_linear(s["x"], s["w"], bias=s["bias"], act=c["act"], residual=s["residual"],
                               x_scale=s["x_scale"], w_scale=s["w_scale"], out_dtype=s["dtype"])
    y, pre = layer.tg_linear(s["x"], s["w"], bias=s["bias"], act=c["act"], residual=s["residual"], keep_pre=True)
    dx, dw, db = layer.tg_linear_grad(s["dy"], s["x"], s["w"], pre=pre, act=c["act"], bias_grad=c["bias"])
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _own_norm(s):
    from paper_2606_16907_amd import layer
    c = s["case"]
    f = layer.tg_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                          out_dtype=E4M3 if c["out"] == "e4m3" else s["x"].dtype)
    out = {"y": f.y, "scale": f.scale, "hidden": f.hidden if c["residual"] else None}
    if c["grad"]:
        out["dx"], out["dweight"] = layer.tg_rms_norm_grad(s["dy"], f.hidden, s["weight"], f.rstd, dhidden=s["dh"])
    return out


def _own_adamw(s):
    s["opt"].step(s["step"], lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY, seed=s["seed"])
    s["step"] += 1
    return _states(s)


def _states(s):
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale")}


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


def _plain_linear(s):
    c, dtype = s["case"], s["dtype"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["x_scale"] is not None:
        z = z * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not c["grad"]:
        return y.to(dtype)
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_grad(z, c["act"])
    return {"y": y.to(dtype), "dx": (dz @ w).to(dtype), "dw": (dz.t() @ x).to(dtype),
            "db": dz.sum(0).to(dtype) if c["bias"] else None}


def _plain_norm(s):
    c, dtype = s["case"], s["x"].dtype
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    w = s["weight"].float()
    y = h * rstd * w
    out = {"y": y.to(dtype), "scale": None, "hidden": h.to(dtype) if c["residual"] else None}
    if c["out"] == "e4m3":
        scale = y.abs().amax(1) / E4M3_MAX
        scale = torch.where(scale > 0, scale, torch.ones_like(scale))
        out["y"], out["scale"] = (y / scale[:, None]).to(E4M3), scale
    if c["grad"]:
        dy = s["dy"].float()
        g = dy * w
        dx = rstd * (g - h * rstd * rstd * (g * h).mean(1, keepdim=True))
        out["dx"] = (dx + s["dh"].float() if s["dh"] is not None else dx).to(dtype)
        out["dweight"] = (dy * h * rstd).sum(0).to(dtype)
    return out


def _mix(x):
    """32 mixed bits of 32 bits (held in int64)."""
    x = x ^ (x >> 16)
    x = (x * 0x85A308D3) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xA4093823) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(s):
    """32 random bits of each element, [blocks, BLOCK]."""
    key = _mix((s["seed"] + s["step"] * 0x9E3779B1 + s["tensor"] * 0x13198A2F) & 0xFFFFFFFF)
    element = s["block"][:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    return _mix((element + key[:, None]) & 0xFFFFFFFF)


def _round_e4m3(a, bits16):
    """|a| <= 448 (of a scaled block) to e4m3, up or down by 16 random bits: of the 20 bits that the type does not hold
    the upper 16 are added to; below 2^-6 the values are multiples of 2^-9."""
    mag = a.abs()
    word = (mag.view(torch.int32) + (bits16 << 4).to(torch.int32)) & ~0xFFFFF
    low = torch.floor(mag * 512 + bits16.to(torch.float32) / 65536) / 512
    q = torch.where(mag >= 2.0 ** -6, word.view(torch.float32), low).clamp_max(E4M3_MAX)
    return torch.where(a < 0, -q, q)


def _to_blocks(x, bits16, keep_positive=False):
    most = x.abs().amax(1, keepdim=True)
    fine = most > 1e-30
    a = x * torch.where(fine, E4M3_MAX / most, torch.zeros_like(most))
    q = _round_e4m3(a, bits16)
    if keep_positive:  # a second moment above zero never becomes zero
        q = torch.where((a > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
    return q.to(E4M3), torch.where(fine, most / E4M3_MAX, torch.zeros_like(most))[:, 0]


def _plain_adamw(s):
    eight = s["case"]["bits"] == 8
    g = s["grad"].float()
    m, v = s["m"].float(), s["v"].float()
    if eight:
        m = (m.view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (v.view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    c1, c2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    w = s["master"] * (1 - LR * DECAY) - LR * (m / c1) / (torch.sqrt(v / c2) + ADAM_EPS)
    s["master"].copy_(w)
    s["param"].copy_(w)
    if eight:
        bits = _random_bits(s)
        q, scale = _to_blocks(m.view(-1, BLOCK), bits >> 16)
        s["m"].copy_(q.view(-1)), s["m_scale"].copy_(scale)
        q, scale = _to_blocks(torch.sqrt(v).view(-1, BLOCK), bits & 0xFFFF, keep_positive=True)
        s["v"].copy_(q.view(-1)), s["v_scale"].copy_(scale)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    s["step"] += 1
    return _states(s)


# ----------------------------------------------------------------------------
# work and 64-bit results
# ----------------------------------------------------------------------------
def work(case):
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        e, o = (1, 2) if case["type"] == "e4m3" else (2, 2)
        nbytes = e * (m * k + n * k) + o * m * n * (1 + case["residual"]) + o * n * case["bias"]
        nbytes += 4 * (m + n) if case["type"] == "e4m3" else 0
        flops = 2.0 * m * k * n
        if case["grad"]:  # dy read, dx and dw written, the bias's gradient
            nbytes += o * (m * n + m * k + n * k + n * case["bias"])
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "rms_norm":
        rows, cols, e = case["rows"], case["cols"], 4 if case["type"] == "f32" else 2
        n = rows * cols
        nbytes = e * n * (1 + 2 * case["residual"]) + e * cols + (n + 4 * rows if case["out"] == "e4m3" else e * n)
        flops = 5.0 * n
        if case["grad"]:  # dy and the residual stream's gradient read, dx and the weight's gradient written
            nbytes += e * n * (2 + case["residual"]) + e * cols
            flops += 9.0 * n
        return {"bytes": nbytes, "flops": flops}
    n = sum(_tensor_sizes(case))
    # gradient, weight written, master copy and two moments read and written
    nbytes = n * (2 + 2 + 8 + (4 if case["bits"] == 8 else 16))
    nbytes += 16 * sum(-(-t // BLOCK) for t in _tensor_sizes(case)) if case["bits"] == 8 else 0
    return {"bytes": nbytes, "flops": 16.0 * n}


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"linear": _exact_linear, "rms_norm": _exact_norm, "adamw": _exact_adamw}[case["op"]](s)


def _exact_linear(s):
    c, f64 = s["case"], torch.float64
    x, w = s["x"].to(f64), s["w"].to(f64)
    if s["x_scale"] is not None:
        x, w = x * s["x_scale"].to(f64)[:, None], w * s["w_scale"].to(f64)[:, None]
    z = torch.mm(x, w.t().contiguous())
    if s["bias"] is not None:
        z += s["bias"].to(f64)
    normal = torch.distributions.Normal(torch.zeros((), dtype=f64, device="cuda"), torch.ones((), dtype=f64, device="cuda"))
    if c["act"] == "relu":
        y, slope = torch.maximum(z, torch.zeros_like(z)), torch.where(z > 0, 1.0, 0.0).to(f64)
    elif c["act"] == "silu":
        t = torch.sigmoid(z)
        y, slope = z * t, t + z * t * (1 - t)
    elif c["act"] == "gelu":
        y, slope = z * normal.cdf(z), normal.cdf(z) + z * torch.exp(normal.log_prob(z))
    else:
        y, slope = z, torch.ones_like(z)
    if s["residual"] is not None:
        y = y + s["residual"].to(f64)
    if not c["grad"]:
        return y
    dz = s["dy"].to(f64) * slope
    return {"y": y, "dx": torch.mm(dz, w), "dw": torch.mm(dz.t().contiguous(), x),
            "db": dz.sum(0) if c["bias"] else None}


def _exact_norm(s):
    c, f64 = s["case"], torch.float64
    h = s["x"].to(f64)
    if s["residual"] is not None:
        h = h + s["residual"].to(f64)
    var = h.square().sum(1) / h.shape[1] + EPS
    xhat = h / var.sqrt()[:, None]
    w = s["weight"].to(f64)
    out = {"y": xhat * w, "scale": None, "hidden": h if c["residual"] else None}
    if c["out"] == "e4m3":
        out["scale"] = out["y"].abs().amax(1) / E4M3_MAX
        out["y"] = out["y"] / out["scale"][:, None]
    if c["grad"]:
        dy = s["dy"].to(f64)
        g = dy * w
        dx = (g - xhat * (g * xhat).mean(1, keepdim=True)) / var.sqrt()[:, None]
        out["dx"] = dx if s["dh"] is None else dx + s["dh"].to(f64)
        out["dweight"] = (dy * xhat).sum(0)
    return out


def _exact_adamw(s):
    f64, eight = torch.float64, s["case"]["bits"] == 8
    g, m, v, w = (s[k].to(f64) for k in ("grad", "m", "v", "master"))
    if eight:
        m = m * s["m_scale"].to(f64).repeat_interleave(BLOCK)
        v = (v * s["v_scale"].to(f64).repeat_interleave(BLOCK)).square()
    m = m + (g - m) * (1 - BETA1)
    v = v + (g.square() - v) * (1 - BETA2)
    del g
    rate = LR / (1 - BETA1 ** s["step"])
    w = w - LR * DECAY * w - rate * m / ((v / (1 - BETA2 ** s["step"])).sqrt() + ADAM_EPS)
    out = {"param": w, "master": w, "m": m, "v": v, "m_scale": None, "v_scale": None}
    if eight:  # the codes are rounded at random: only their scales have a value
        out.update(m=None, v=None, m_scale=m.abs().view(-1, BLOCK).amax(1) / E4M3_MAX,
                   v_scale=v.view(-1, BLOCK).amax(1).sqrt() / E4M3_MAX)
    return out
