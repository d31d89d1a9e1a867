"""AdamW over many tensors against 64 bits, its 8-bit states' rounding among it."""
import math

import numpy as np
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E4M3, E32, U

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
RATES = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-8, weight_decay=0.1)
SIZES = [1, 3, 255, 256, 257, 4095, 4096, 4097, 10000, 0, 77777]


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def flat(gen, n, dtype, std=1.0, offset=0):
    return (torch.randn(n + offset, generator=gen) * std).to(dtype).cuda()[offset:]


def plain(w, g, m, v, step, gs=1.0, lr=0.0, beta1=0.0, beta2=0.0, eps=0.0, weight_decay=0.0):
    g = g * gs
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    upd = (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps)
    return w - lr * weight_decay * w - lr * upd, m, v, upd


@pytest.mark.parametrize("param,grad,master", [(F32, F32, False), (BF16, BF16, True), (BF16, F32, True), (BF16, BF16, False),
                                               (F16, F16, True), (F16, F32, False)])
@pytest.mark.parametrize("offset", [0, 1])
def test_steps_with_32_bit_states(param, grad, master, offset):
    gen = R.generator(param, grad, master, offset)
    p = [flat(gen, n, param, 0.5, offset) for n in SIZES]
    g = [flat(gen, n, grad, 0.01, offset) for n in SIZES]
    m = [flat(gen, n, F32, 0.01, offset) for n in SIZES]
    v = [flat(gen, n, F32, 0.01, offset).square() for n in SIZES]
    w = [t.float() + (flat(gen, t.numel(), F32, 1e-3) if master else 0) for t in p]
    opt = layer().AdamW(p, g, m, v, masters=w if master else None)
    for step in (1, 2, 1000):
        before = [[R.f64(t) for t in s] for s in (w if master else p, g, m, v)]
        opt.step(step, grad_scale=0.5, **RATES)
        for i, n in enumerate(SIZES):
            want, wm, wv, upd = plain(*(s[i] for s in before), step, 0.5, **RATES)
            size = before[2][i].abs() + before[1][i].abs()
            em = 4 * E32 * size
            ev = 4 * E32 * (before[3][i] + before[1][i].square())
            R.within(m[i], wm, em, f"m {i}")
            R.within(v[i], wv, ev + 1e-37, f"v {i}")
            # m may cancel; the root and the quotient are good to a few units, the rates are rounded to 32 bits
            c = (1 - RATES["beta2"] ** step) ** 0.5 / (1 - RATES["beta1"] ** step)
            ew = RATES["lr"] * (12 * E32 * upd.abs() + em * c / (wv.sqrt() + 1e-12) + upd.abs() * ev / (wv + 1e-30)) + 3 * E32 * want.abs() + 1e-37
            if master:
                R.within(w[i], want, ew, f"master {i}")
                assert torch.equal(p[i], w[i].to(param)), i
            else:
                R.within(p[i], want, ew + 1.01 * U[param] * want.abs() + (2.0 ** -25 if param == F16 else 0), f"param {i}")


def mix(x):
    x = (x ^ (x >> np.uint64(16))) & np.uint64(0xFFFFFFFF)
    x = (x * np.uint64(0x85A308D3)) & np.uint64(0xFFFFFFFF)
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0xA4093823)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def bits_of(n, tensor, step, seed):
    key = mix(np.array([(seed + step * 0x9E3779B1 + tensor * 0x13198A2F) % (1 << 32)], dtype=np.uint64))
    return mix((np.arange(n, dtype=np.uint64) + key) & np.uint64(0xFFFFFFFF))


def neighbours(a):
    """The e4m3 values at or below and at or above |a| <= 448."""
    a = np.minimum(np.abs(a), 448.0)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 1e-30))), -6) - 3)
    return np.floor(a / step) * step, np.ceil(a / step) * step, step


def blocks_max(x):
    n = len(x)
    padded = np.zeros(-(-n // 256) * 256)
    padded[:n] = np.abs(x)
    return padded.reshape(-1, 256).max(1)


def dequantised(codes, scale):
    n = codes.numel()
    return R.f64(codes.float()) * R.f64(scale).repeat_interleave(256)[:n]


def states8(gen, sizes, offset=0):
    L = layer()
    m, v, ms, vs = [], [], [], []
    for n in sizes:
        for codes, scales, x in ((m, ms, flat(gen, n, F32, 0.01)), (v, vs, flat(gen, n, F32, 0.01).abs() + 1e-4)):
            most = torch.from_numpy(blocks_max(x.cpu().double().numpy())).float().cuda()
            scales.append(most / 448)
            q = torch.empty(n + offset, dtype=torch.uint8, device="cuda").view(E4M3)[offset:]
            q.copy_((x / scales[-1].repeat_interleave(256)[:n]).to(E4M3))
            codes.append(q)
    return m, v, ms, vs


@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("param,master", [(BF16, True), (F32, False)])
def test_a_step_with_8_bit_states(param, master, offset):
    """The step is the 32-bit one from the states' values; the new states lie on one of the two neighbours of the new
    moments, on the one that the given random bits say wherever 32-bit errors leave no doubt."""
    gen = R.generator("eight", param, offset)
    p = [flat(gen, n, param, 0.5, offset) for n in SIZES]
    g = [flat(gen, n, param, 0.01, offset) for n in SIZES]
    m, v, ms, vs = states8(gen, SIZES, offset)
    w = [t.float() for t in p]
    step, seed = 7, 0xDEADBEEF
    old = [(R.f64(w[i] if master else p[i]), R.f64(g[i]), dequantised(m[i], ms[i]), dequantised(v[i], vs[i]).square())
           for i in range(len(SIZES))]
    layer().AdamW(p, g, m, v, ms, vs, masters=w if master else None).step(step, seed=seed, **RATES)
    for i, n in enumerate(SIZES):
        want, wm, wv, upd = plain(*old[i], step, **RATES)
        em = 6 * E32 * (old[i][2].abs() + old[i][1].abs())
        c = (1 - RATES["beta2"] ** step) ** 0.5 / (1 - RATES["beta1"] ** step)
        ew = RATES["lr"] * (24 * E32 * upd.abs() + em * c / (wv.sqrt() + 1e-12)) + 3 * E32 * want.abs()
        R.within(w[i] if master else p[i], want, ew, f"w {i}")
        if n == 0:
            continue
        bits = bits_of(n, i, step, seed)
        for codes, scales, x, share, positive in ((m[i], ms[i], wm, bits >> np.uint64(16), False),
                                                  (v[i], vs[i], wv.sqrt(), bits & np.uint64(0xFFFF), True)):
            x = x.numpy()
            most = blocks_max(x)
            assert np.allclose(scales.cpu().numpy(), most / 448, rtol=1e-6, atol=0)
            a = x / (np.repeat(most, 256)[:n] / 448)
            low, high, unit = neighbours(a)
            got = np.abs(codes.float().cpu().numpy().astype(np.float64))
            assert ((got == low) | (got == high) | (np.abs(got - np.abs(a)) <= unit * 1e-3)).all() or positive
            frac = (np.abs(a) - low) / unit
            up = frac + share.astype(np.float64) / 65536 >= 1
            # 16 of the 20 bits are added to: doubt within 2^-16 of a step, and within 32-bit errors of a
            sure = np.abs(frac + share.astype(np.float64) / 65536 - 1) > 2.0 ** -15 + 64 * E32 * np.maximum(np.abs(a) / unit, 1)
            sure &= frac > 1e-4
            picked = np.where(up, np.minimum(low + unit, 448.0), low)
            if positive:
                picked = np.where((picked == 0) & (a > 0), 2.0 ** -9, picked)
                assert (codes.float().cpu().numpy() > 0).all()
            assert sure.mean() > 0.9 or n < 100
            assert (got[sure] == picked[sure]).all(), (i, int((got[sure] != picked[sure]).sum()))


def test_8_bit_states_follow_the_mean():
    """Gradients of one size for 400 steps: v goes where 32-bit states go, which rounding to nearest would prevent."""
    L = layer()
    n = 1 << 16
    p = [torch.zeros(n, device="cuda")]
    g = [torch.full((n,), 0.01, device="cuda")]
    m, v, ms, vs = L.adamw_states(p, bits=8)
    ms[0].fill_(0.02 / 448), vs[0].fill_(0.02 / 448)  # both begin at twice their limit
    m[0].copy_(torch.full((n,), 448.0, device="cuda").to(E4M3)), v[0].copy_(m[0])
    opt = L.AdamW(p, g, m, v, ms, vs)
    for step in range(1, 401):
        opt.step(step, lr=0.0, beta1=0.9, beta2=0.99, seed=step)
    root = dequantised(v[0], vs[0])
    want = math.sqrt(1e-4 + (4e-4 - 1e-4) * 0.99 ** 400)
    # rounding up and down adds the variance of a step's rounding to v: about 4% in sqrt(v) at most with these betas
    assert abs(float(root.mean()) / want - 1) < 0.05, float(root.mean()) / want
    assert abs(float(dequantised(m[0], ms[0]).mean()) / 0.01 - 1) < 0.02


def test_values_that_are_not_finite_stay_alone():
    L = layer()
    for bits in (32, 8):
        n = 1000
        p, g = [torch.ones(n, device="cuda")], [torch.full((n,), 0.01, device="cuda")]
        g[0][300], g[0][700] = float("nan"), float("inf")
        states = L.adamw_states(p, bits=bits)
        L.AdamW(p, g, *states).step(1, lr=0.01)
        bad = torch.zeros(n, dtype=torch.bool, device="cuda")
        bad[300] = bad[700] = True
        assert torch.equal(~torch.isfinite(states[0][0].float()), bad)
        assert torch.equal(~torch.isfinite(states[1][0].float()), bad)
        assert bool(torch.isfinite(p[0][~bad]).all()) and bool((p[0][~bad] < 1).all())


def test_zero_gradients_and_zero_states():
    L = layer()
    for bits in (32, 8):
        p, g = [torch.full((600,), 2.0, device="cuda")], [torch.zeros(600, device="cuda")]
        states = L.adamw_states(p, bits=bits)
        L.AdamW(p, g, *states).step(1, lr=0.01, weight_decay=0.5)
        assert bool(((p[0] - 1.99).abs() < 1e-6).all())
        assert all(bool((s[0].float() == 0).all()) for s in states)


def test_many_short_tensors_other_streams_and_new_gradients():
    L = layer()
    gen = R.generator("short")
    sizes = [int(x) for x in torch.randint(0, 300, (500,), generator=gen)]
    p, g = [flat(gen, n, F32) for n in sizes], [flat(gen, n, F32) for n in sizes]
    m, v = L.adamw_states(p)
    old, opt = [t.clone() for t in p], L.AdamW(p, g, m, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt.step(1, lr=0.25, eps=0.0)
    side.synchronize()
    for a, b, d in zip(old, p, g):  # the first step moves every weight by lr against its gradient's sign
        assert torch.allclose(a - b, 0.25 * d.sign(), atol=1e-6)
    other = [torch.zeros_like(t) for t in g]
    opt.set_grads(other)
    del g
    was = [t.clone() for t in m]
    opt.step(2, lr=0.0)
    assert all(torch.allclose(b, 0.9 * a) for a, b in zip(was, m))
    opt.close()
    with pytest.raises(ValueError, match="closed"):
        opt.step(3, lr=0.0)


def test_graph_replays():
    L = layer()
    gen = R.generator("graph")
    p, g = [flat(gen, 5000, F32)], [flat(gen, 5000, F32)]
    q = [p[0].clone()]
    a, b = L.adamw_states(p, bits=8), L.adamw_states(q, bits=8)
    one, two = L.AdamW(p, g, *a), L.AdamW(q, g, *b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step(5, lr=1e-2, seed=3)
    for k in range(3):
        graph.replay()
        two.step(5, lr=1e-2, seed=3)
        torch.cuda.synchronize()
        assert torch.equal(p[0], q[0]) and all(torch.equal(x[0].view(torch.uint8), y[0].view(torch.uint8)) for x, y in zip(a, b))


def test_refusals():
    L = layer()
    from paper_2606_16907_amd.tangram import TangramError
    t = torch.zeros(64, device="cuda")
    e = t.to(E4M3)
    s = torch.zeros(1, device="cuda")
    bad = [lambda: L.AdamW([t], [t.half()], [t], [t]), lambda: L.AdamW([t], [t], [t], [t[:3]]), lambda: L.AdamW([t], [t], [t], []),
           lambda: L.AdamW([t[::2]], [t[:32]], [t[:32]], [t[:32]]), lambda: L.AdamW([t], [t], [e], [e]),
           lambda: L.AdamW([t], [t], [t], [t], [s], [s]), lambda: L.AdamW([t], [t], [e], [e], [s], [t]),
           lambda: L.AdamW([t], [t], [t], [e]), lambda: L.AdamW([t.cpu()], [t], [t], [t]), lambda: L.AdamW([t.double()], [t], [t], [t])]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {k} was taken")
    with pytest.raises(TangramError, match="master"):
        L.AdamW([t], [t], [t.clone()], [t.clone()], masters=[t.clone()])
    opt = L.AdamW([t], [t.clone()], [t.clone()], [t.clone()])
    for kw, word in ((dict(step=0, lr=1.0), "step"), (dict(step=1, lr=float("nan")), "finite"), (dict(step=1, lr=1.0, beta1=1.0), "beta"),
                     (dict(step=1, lr=1.0, grad_scale=float("inf")), "finite")):
        with pytest.raises(TangramError, match=word):
            opt.step(**kw)
