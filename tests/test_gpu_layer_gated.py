"""The gated projections and their gradients against 64 bits."""
import pytest
import torch

from tests import gated_ref as G
from tests import layer_ref as R
from tests.layer_ref import E4M3

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
ACTS = ["silu", "none", "relu", "gelu"]


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def quantised(t):
    scale = (t.abs().amax(1) / 448).clamp_min(1e-12)
    return (t / scale[:, None]).to(E4M3), scale


def biases(gen, n, dtype):
    return [R.rows(gen, 1, n, dtype, std=0.5)[0] for _ in range(2)]


SIZES = [(1, 1, 1), (1, 64, 8), (2, 40, 9), (3, 72, 33), (5, 513, 7), (8, 256, 130), (9, 64, 128), (16, 96, 65), (33, 129, 31), (63, 200, 127),
         (64, 1000, 128), (65, 257, 129), (127, 64, 64), (129, 1030, 191), (300, 264, 257), (513, 72, 520)]


@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype, pad):
    gen = R.generator("gated", m, k, n, dtype, pad)
    name = ACTS[(m + k + n + pad) % 4]
    x, wg, wu = R.rows(gen, m, k, dtype, pad), R.rows(gen, n, k, dtype, 0, k ** -0.5), R.rows(gen, n, k, dtype, pad, k ** -0.5)
    bg, bu = biases(gen, n, dtype) if (m + n) % 2 else (None, None)
    y, gate, up = layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act=name, keep_pre=True)
    want = G.projections(x, wg, wu, bg, bu)
    R.within(gate, *G.kept(*want[0], dtype), "gate")
    R.within(up, *G.kept(*want[1], dtype), "up")
    R.within(y, *G.forward(*want, name, dtype), "y")
    assert torch.equal(y, layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act=name))


@pytest.mark.parametrize("m,k,n", [(1, 16, 1), (1, 8192, 40), (4, 300, 129), (9, 160, 70), (48, 4096, 200), (64, 777, 65), (65, 777, 65), (130, 1000, 300)])
@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("out", [BF16, F16])
def test_forward_in_8_bits(m, k, n, pad, out):
    gen = R.generator("gated8", m, k, n, pad)
    x, sx = quantised(R.rows(gen, m, k, torch.float32))
    wide = torch.zeros(m, k + pad, dtype=torch.uint8, device="cuda").view(E4M3)
    wide[:, :k] = x
    x = wide[:, :k]
    (wg, sg), (wu, su) = (quantised(R.rows(gen, n, k, torch.float32, std=k ** -0.5)) for _ in range(2))
    bg, bu = biases(gen, n, out) if pad else (None, None)
    y = layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act="silu", x_scale=sx, gate_scale=sg, up_scale=su, out_dtype=out)
    want = G.projections(x, wg, wu, bg, bu, sx, sg, su)
    R.within(y, *G.forward(*want, "silu", out), "y")


@pytest.mark.parametrize("m,k,n,pad,dtype", [(1, 8192, 9, 0, BF16), (1, 14336, 640, 0, BF16), (4, 10803, 345, 3, F16), (8, 14336, 512, 0, BF16),
                                             (600, 6000, 300, 0, F16), (1500, 8200, 1500, 0, BF16), (3500, 1000, 2041, 8, BF16),
                                             (16, 4096, 5000, 0, BF16), (24, 2048, 4500, 0, F16), (50, 4100, 1030, 2, BF16), (4352, 2056, 2176, 0, BF16), (4200, 1000, 4100, 3, F16), (4352, 4104, 2176, 0, BF16)])
def test_shared_sums_and_large_tiles(m, k, n, pad, dtype):
    gen = R.generator("gated large", m, k, n, pad)
    x, wg, wu = R.rows(gen, m, k, dtype, pad), R.rows(gen, n, k, dtype, pad, k ** -0.5), R.rows(gen, n, k, dtype, 0, k ** -0.5)
    bg, bu = biases(gen, n, dtype)
    y = layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act="gelu")
    R.within(y, *G.forward(*G.projections(x, wg, wu, bg, bu), "gelu", dtype), "y")


GRAD_SIZES = [(1, 1, 1), (1, 40, 24), (2, 17, 129), (16, 64, 64), (37, 100, 72), (64, 128, 256), (100, 1, 33), (129, 257, 65), (256, 256, 192),
              (300, 264, 520), (513, 72, 300), (1030, 130, 70)]


@pytest.mark.parametrize("pad", [0, 5, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,k,n", GRAD_SIZES)
def test_gradients(m, k, n, dtype, pad):
    gen = R.generator("gated grad", m, k, n, dtype, pad)
    name = ACTS[(m + k + n + pad) % 4]
    x, wg, wu = R.rows(gen, m, k, dtype, pad), R.rows(gen, n, k, dtype, pad, k ** -0.5), R.rows(gen, n, k, dtype, 0, k ** -0.5)
    dy, gate, up = R.rows(gen, m, n, dtype, pad), R.rows(gen, m, n, dtype, 0, 1.5), R.rows(gen, m, n, dtype, pad, 1.5)
    got = layer().tg_gated_grad(dy, x, wg, wu, gate, up, act=name, bias_grad=True)
    for key, want in G.grads(dy, x, wg, wu, gate, up, name).items():
        R.within(getattr(got, key), *want, key)


@pytest.mark.parametrize("m,k,n", [(300, 3400, 8200), (8200, 1500, 700), (2048, 520, 2050), (4352, 4352, 1024)])
def test_gradients_of_large_tiles_and_shared_sums(m, k, n):
    gen = R.generator("gated large grad", m, k, n)
    x, wg, wu = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16, 0, k ** -0.5), R.rows(gen, n, k, BF16, 0, k ** -0.5)
    dy, gate, up = (R.rows(gen, m, n, BF16) for _ in range(3))
    got = layer().tg_gated_grad(dy, x, wg, wu, gate, up, act="silu", bias_grad=True)
    for key, want in G.grads(dy, x, wg, wu, gate, up, "silu").items():
        R.within(getattr(got, key), *want, key)


def test_each_gradient_alone():
    L, gen = layer(), R.generator("alone")
    m, k, n = 70, 136, 100
    x, wg, wu = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16), R.rows(gen, n, k, BF16)
    dy, gate, up = (R.rows(gen, m, n, BF16) for _ in range(3))
    every = L.tg_gated_grad(dy, x, wg, wu, gate, up, bias_grad=True)
    alone = L.tg_gated_grad(dy, x, wg, wu, gate, up, w_grad=False)
    assert torch.equal(alone.dx, every.dx) and alone[1:] == (None,) * 4
    alone = L.tg_gated_grad(dy, x, wg, wu, gate, up, x_grad=False)
    assert alone.dx is None and torch.equal(alone.dw_gate, every.dw_gate) and torch.equal(alone.dw_up, every.dw_up)
    alone = L.tg_gated_grad(dy, x, wg, wu, gate, up, x_grad=False, w_grad=False, bias_grad=True)
    assert torch.equal(alone.dgate_bias, every.dgate_bias) and torch.equal(alone.dup_bias, every.dup_bias)
    # one weight's gradient and one bias's, through the C entry
    import ctypes
    lib = L.load_library()
    for gate_only in (True, False):
        dw, db = torch.zeros_like(wg), torch.zeros_like(dy[0])
        ptr = [t.data_ptr() for t in (dy, gate, up, x, wg, wu)]
        outs = [None, dw.data_ptr() if gate_only else None, None if gate_only else dw.data_ptr(),
                db.data_ptr() if gate_only else None, None if gate_only else db.data_ptr()]
        a = L.TgGatedGradArgs(*ptr, *outs, m, n, k, n, n, n, k, k, k, k, k, k, 1, L.ACTS["silu"])
        ws = torch.empty(lib.tg_gated_grad_workspace_bytes(a), dtype=torch.uint8, device="cuda")
        assert lib.tg_gated_grad(ctypes.byref(a), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(dw, every.dw_gate if gate_only else every.dw_up)
        assert torch.equal(db, every.dgate_bias if gate_only else every.dup_bias)


@pytest.mark.parametrize("name", ["silu", "gelu", "none"])
def test_gradients_against_differences(name):
    """Central differences of the loss sum(dy y) in 64 bits: their own error is h^2 / 6 times a third derivative of order
    10 at these sizes, far below the bound.  gate and up are kept in 16 bits: the slope and the value move by at most
    0.8 and 1.13 times 2^-8 |gate|, up by 2^-8 |up|."""
    gen = R.generator("gated differences", name)
    m, k, n, h = 5, 12, 9, 1e-4
    x, wg, wu = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16, std=k ** -0.5), R.rows(gen, n, k, BF16, std=k ** -0.5)
    bg, bu = biases(gen, n, BF16)
    dy = R.rows(gen, m, n, BF16)
    _, gate, up = layer().tg_gated(x, wg, wu, gate_bias=bg, up_bias=bu, act=name, keep_pre=True)
    got = layer().tg_gated_grad(dy, x, wg, wu, gate, up, act=name, bias_grad=True)
    at = {"dx": R.f64(x), "dw_gate": R.f64(wg), "dw_up": R.f64(wu), "dgate_bias": R.f64(bg), "dup_bias": R.f64(bu)}
    d = R.f64(dy)

    def both():
        return at["dx"] @ at["dw_gate"].t() + at["dgate_bias"], at["dx"] @ at["dw_up"].t() + at["dup_bias"]

    def loss():
        g, u = both()
        return float((d * R.act(g, name) * u).sum())

    g, u = both()
    bounds = G.grads(dy, x, wg, wu, g.to(BF16), u.to(BF16), name)
    moved_g = d.abs() * 2.0 ** -8 * u.abs() * (0.8 * g.abs() + 1.13)
    moved_u = d.abs() * 2.0 ** -8 * 1.13 * g.abs()
    extra = {"dx": moved_g @ at["dw_gate"].abs() + moved_u @ at["dw_up"].abs(), "dw_gate": moved_g.t() @ at["dx"].abs(),
             "dw_up": moved_u.t() @ at["dx"].abs(), "dgate_bias": moved_g.sum(0), "dup_bias": moved_u.sum(0)}
    for key, t in at.items():
        flat, grad = t.reshape(-1), R.f64(getattr(got, key)).reshape(-1)
        for i in range(0, flat.numel(), 3):
            keep = float(flat[i])
            flat[i] = keep + h
            above = loss()
            flat[i] = keep - h
            below = loss()
            flat[i] = keep
            far = abs((above - below) / (2 * h) - float(grad[i]))
            assert far <= float((bounds[key][1] + 2 * extra[key]).reshape(-1)[i]) + 1e-6, (key, i, far)


@pytest.mark.parametrize("m,k,n", [(0, 8, 8), (4, 0, 8), (4, 8, 0), (300, 0, 300)])
def test_empty_sizes(m, k, n):
    L = layer()
    x, wg = torch.ones(m, k, device="cuda", dtype=BF16), torch.ones(n, k, device="cuda", dtype=BF16)
    bias, dy = torch.full((n,), 2.0, device="cuda", dtype=BF16), torch.ones(m, n, device="cuda", dtype=BF16)
    y, gate, up = L.tg_gated(x, wg, wg, gate_bias=bias, up_bias=bias, act="relu", keep_pre=True)
    assert y.shape == (m, n) and bool((y == (2 + k) ** 2).all())
    g = L.tg_gated_grad(dy, x, wg, wg, gate, up, act="relu", bias_grad=True)
    assert bool((g.dx == 2 * n * (2 + k)).all()) and bool((g.dw_gate == m * (2 + k)).all()) and bool((g.dup_bias == m * (2 + k)).all())


@pytest.mark.parametrize("m", [1, 40, 300])
def test_nan_and_infinity_stay_in_their_rows_and_columns(m):
    """Bytes past a row's end must not reach a result: what lies there is NaN."""
    L, gen = layer(), R.generator("gated nan", m)
    for k, pad in ((72, 8), (70, 10), (69, 3), (64, 64)):
        x, wg, wu = R.rows(gen, m, k, BF16, pad), R.rows(gen, 90, k, BF16, pad), R.rows(gen, 90, k, BF16, pad)
        for t in (x, wg, wu):
            t.as_strided((t.shape[0] - 1, pad), t.stride(), t.storage_offset() + k).fill_(float("nan"))
        assert bool(torch.isfinite(L.tg_gated(x, wg, wu)).all())
        x[m // 2, k - 1] = float("nan")
        wg[3, 0] = float("nan")
        wu[70, k - 1] = float("nan")
        bad = ~torch.isfinite(L.tg_gated(x, wg, wu))
        want = torch.zeros_like(bad)
        want[m // 2], want[:, 3], want[:, 70] = True, True, True
        assert torch.equal(bad, want)
        wg[3, 0], wu[70, k - 1], x[m // 2, k - 1] = 1.0, 1.0, 1.0
        dy, gate, up = (R.rows(gen, m, 90, BF16, 6) for _ in range(3))
        for t in (dy, gate, up):
            t.as_strided((m - 1, 6), t.stride(), t.storage_offset() + 90).fill_(float("nan"))
        assert all(bool(torch.isfinite(t).all()) for t in L.tg_gated_grad(dy, x, wg, wu, gate, up, bias_grad=True))
        gate[m // 2, 80] = float("nan")
        g = L.tg_gated_grad(dy, x, wg, wu, gate, up, bias_grad=True)
        bad = torch.isnan(g.dx)
        want = torch.zeros_like(bad)
        want[m // 2] = True
        assert torch.equal(bad, want)
        for t in (g.dw_gate, g.dw_up):
            bad = torch.isnan(t)
            want = torch.zeros_like(bad)
            want[80] = True
            assert torch.equal(bad, want)
        assert torch.isnan(g.dgate_bias).nonzero().flatten().tolist() == [80]


def test_pre_activations_that_are_infinities():
    """A gate beyond 16 bits is kept as an infinity: the slope and the value are the activation's limits there."""
    L = layer()
    x, w = torch.ones(1, 8, device="cuda", dtype=BF16), torch.eye(2, 8, device="cuda", dtype=BF16)
    gate = torch.tensor([[float("-inf"), float("inf")]], device="cuda", dtype=BF16)
    up, dy = torch.ones(1, 2, device="cuda", dtype=BF16), torch.ones(1, 2, device="cuda", dtype=BF16)
    for name in ("silu", "gelu", "relu"):
        g = L.tg_gated_grad(dy, x, w, w, gate, up, act=name, bias_grad=True)
        assert g.dgate_bias.tolist() == [0.0, 1.0] and g.dup_bias.tolist() == [0.0, float("inf")], name


def test_gradients_of_large_pre_activations():
    """Where exp(-z) or exp(-z^2 / 2) leave 32 bits the slopes and values are 0 below, 1 and z above."""
    L, gen = layer(), R.generator("large gates")
    z = torch.tensor([-3e4, -1000.0, -200.0, -128.5, -127.0, -89.0, -20.0, 20.0, 89.0, 128.5, 1000.0, 3e4])
    m, n, k = 5, len(z), 24
    gate, up, dy = z.repeat(m, 1).to(F16).cuda(), R.rows(gen, m, n, F16), R.rows(gen, m, n, F16, std=2.0 ** -8)
    x, wg, wu = R.rows(gen, m, k, F16), R.rows(gen, n, k, F16), R.rows(gen, n, k, F16)
    for name in ACTS:
        got = L.tg_gated_grad(dy, x, wg, wu, gate, up, act=name, bias_grad=True)
        for key, want in G.grads(dy, x, wg, wu, gate, up, name).items():
            R.within(getattr(got, key), *want, f"{name} {key}")


def test_8_bits_without_scales_and_kept():
    L, gen = layer(), R.generator("no scales")
    for m in (3, 150):
        x, wg, wu = (R.rows(gen, r, 200, torch.float32).to(E4M3) for r in (m, 90, 90))
        y, gate, up = L.tg_gated(x, wg, wu, act="gelu", keep_pre=True)
        one = [torch.ones(r, device="cuda") for r in (m, 90, 90)]
        want = G.projections(x, wg, wu, None, None, *one)
        R.within(gate, *G.kept(*want[0], BF16), "gate")
        R.within(up, *G.kept(*want[1], BF16), "up")
        R.within(y, *G.forward(*want, "gelu", BF16), "y")


def test_halves_of_one_weight_and_outputs_that_are_given():
    L, gen = layer(), R.generator("halves")
    m, k, n = 140, 200, 104
    x, w = R.rows(gen, m, k, BF16), R.rows(gen, 2 * n, k, BF16, std=k ** -0.5)
    out = torch.zeros(m, n + 4, dtype=BF16, device="cuda")[:, :n]
    y, gate, up = L.tg_gated(x, w[:n], w[n:], keep_pre=True, out=out)
    assert y is out and torch.equal(y, L.tg_gated(x, w[:n].clone(), w[n:].clone()))
    dw, db, dy = torch.empty_like(w), torch.empty(2 * n, dtype=BF16, device="cuda"), R.rows(gen, m, n, BF16)
    g = L.tg_gated_grad(dy, x, w[:n], w[n:], gate, up, bias_grad=True, dw_gate=dw[:n], dw_up=dw[n:], dgate_bias=db[:n], dup_bias=db[n:])
    h = L.tg_gated_grad(dy, x, w[:n].clone(), w[n:].clone(), gate, up, bias_grad=True)
    assert torch.equal(g.dx, h.dx) and torch.equal(dw, torch.cat([h.dw_gate, h.dw_up])) and torch.equal(db, torch.cat([h.dgate_bias, h.dup_bias]))


def test_rows_further_apart_than_32_bits_reach():
    L, gen = layer(), R.generator("gated far")
    m, k, n, ld = 3, 72, 40, 1 << 30
    small, wg, wu = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16), R.rows(gen, n, k, BF16)
    far = torch.empty(2 * ld + 128, dtype=BF16, device="cuda")
    x, out = far.as_strided((m, k), (ld, 1)), far.as_strided((m, n), (ld, 1), 128 - n)
    x.copy_(small)
    want = L.tg_gated(small, wg, wu)
    assert torch.equal(L.tg_gated(x, wg, wu, out=out), want)
    dy, gate, up = (R.rows(gen, m, n, BF16) for _ in range(3))
    a = L.tg_gated_grad(dy, small, wg, wu, gate, up, bias_grad=True)
    out.copy_(gate)
    b = L.tg_gated_grad(dy, x, wg, wu, out, up, bias_grad=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_repeatable_replayed_and_on_another_stream():
    L, gen = layer(), R.generator("gated graph")
    x, wg, wu = R.rows(gen, 200, 512, BF16), R.rows(gen, 320, 512, BF16, std=1 / 16), R.rows(gen, 320, 512, BF16, std=1 / 16)
    dy = R.rows(gen, 200, 320, BF16)

    def step():
        y, gate, up = L.tg_gated(x, wg, wu, act="gelu", keep_pre=True)
        return (y, *L.tg_gated_grad(dy, x, wg, wu, gate, up, act="gelu", bias_grad=True), L.tg_gated(x[:1], wg, wu))

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(R.rows(gen, 200, 512, BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), k


def test_refusals():
    L = layer()
    x, w = torch.zeros(4, 8, device="cuda", dtype=BF16), torch.zeros(6, 8, device="cuda", dtype=BF16)
    dy, one = torch.zeros(4, 6, device="cuda", dtype=BF16), torch.ones(6, device="cuda")
    bad = [lambda: L.tg_gated(x.float(), w, w), lambda: L.tg_gated(x, w, w.half()), lambda: L.tg_gated(x, w, w[:5]),
           lambda: L.tg_gated(x, w[:, :7], w), lambda: L.tg_gated(x.cpu(), w, w), lambda: L.tg_gated(x, w, w, act="tanh"),
           lambda: L.tg_gated(x, w, w, gate_bias=x[0]), lambda: L.tg_gated(x, w, w, x_scale=one[:4], gate_scale=one, up_scale=one),
           lambda: L.tg_gated(x.to(E4M3), w.to(E4M3), w.to(E4M3), gate_scale=one, up_scale=one), lambda: L.tg_gated(x, w, w, out=x),
           lambda: L.tg_gated(x[:1].expand(4, 8), w, w), lambda: L.tg_gated_grad(x, x, w, w, dy, dy),
           lambda: L.tg_gated_grad(dy, x, w, w, dy, dy.float()), lambda: L.tg_gated_grad(dy, x, w, w[:, :4], dy, dy)]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {k} was taken")
    from paper_2606_16907_amd.tangram import TangramError
    with pytest.raises(TangramError, match="workspace"):
        L.tg_gated_grad(dy, x, w, w, dy, dy, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
