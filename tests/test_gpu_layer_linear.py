"""The matrix product with its epilogue and its gradients against 64 bits."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E4M3

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def quantised(t):
    scale = (t.float().abs().amax(1) / 448).clamp_min(1e-12)
    return (t.float() / scale[:, None]).to(E4M3), scale


SIZES = [(1, 1, 1), (1, 64, 16), (1, 4096, 257), (2, 8, 3), (3, 1001, 130), (7, 200, 40), (15, 63, 17), (16, 64, 64), (17, 65, 127),
         (31, 136, 1000), (33, 512, 96), (64, 128, 128), (65, 1000, 65), (127, 72, 300), (128, 256, 128), (129, 257, 129),
         (200, 2048, 72), (255, 320, 513), (256, 64, 256), (257, 192, 264), (300, 4104, 520), (513, 96, 1030)]


@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype, pad):
    gen = R.generator(m, k, n, dtype, pad)
    name = ["none", "relu", "silu", "gelu"][(m + k + n + pad) % 4]
    x, w = R.rows(gen, m, k, dtype, pad), R.rows(gen, n, k, dtype, pad, k ** -0.5)
    bias = R.rows(gen, 1, n, dtype)[0] if (m + n) % 2 else None
    residual = R.rows(gen, m, n, dtype, pad) if (k + n) % 3 else None
    y, pre = layer().tg_linear(x, w, bias=bias, act=name, residual=residual, keep_pre=True)
    want, z, bound = R.linear(x, w, bias, name, residual)
    R.within(y, want, R.linear_bound(want, z, bound, dtype, residual), "y")
    if name == "none":
        assert pre is None
    else:
        R.within(pre, z, R.linear_bound(z, z, bound, dtype), "pre")


@pytest.mark.parametrize("m,k,n", [(1, 16, 8), (1, 8192, 130), (4, 1040, 96), (16, 128, 64), (17, 144, 100), (48, 2048, 72), (64, 31, 9),
                                   (129, 1000, 257), (256, 256, 256), (300, 4112, 264)])
@pytest.mark.parametrize("out", [BF16, F16])
def test_forward_in_8_bits(m, k, n, out):
    gen = R.generator("e4m3", m, k, n)
    x, sx = quantised(R.rows(gen, m, k, torch.float32))
    w, sw = quantised(R.rows(gen, n, k, torch.float32, std=k ** -0.5))
    bias, residual = R.rows(gen, 1, n, out)[0], R.rows(gen, m, n, out, 5)
    y = layer().tg_linear(x, w, bias=bias, act="gelu", residual=residual, x_scale=sx, w_scale=sw, out_dtype=out)
    want, z, bound = R.linear(x, w, bias, "gelu", residual, sx, sw)
    R.within(y, want, R.linear_bound(want, z, bound, out, residual))
    plain = layer().tg_linear(x[:, :k], w, out_dtype=BF16)  # values without scales
    want, z, bound = R.linear(x, w)
    R.within(plain, want, R.linear_bound(want, z, bound, BF16))


@pytest.mark.parametrize("m,k,n,pad", [(1, 10240, 16, 0), (4, 10803, 689, 3), (5, 20483, 33, 5), (8, 14336, 1024, 0), (40, 10247, 100, 1)])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_few_rows_with_long_sums(m, k, n, pad, dtype):
    gen = R.generator("long", m, k, n, pad)
    bias, residual = R.rows(gen, 1, n, BF16)[0], R.rows(gen, m, n, BF16, pad)
    if dtype == E4M3:
        k *= 2
        x, sx = quantised(R.rows(gen, m, k, torch.float32))
        w, sw = quantised(R.rows(gen, n, k, torch.float32, std=k ** -0.5))
    else:
        x, w, sx, sw = R.rows(gen, m, k, BF16, pad), R.rows(gen, n, k, BF16, pad, k ** -0.5), None, None
    y = layer().tg_linear(x, w, bias=bias, act="silu", residual=residual, x_scale=sx, w_scale=sw)
    want, z, bound = R.linear(x, w, bias, "silu", residual, sx, sw)
    R.within(y, want, R.linear_bound(want, z, bound, BF16, residual))


GRAD_SIZES = [(1, 1, 1), (1, 40, 24), (2, 17, 129), (16, 64, 64), (37, 100, 72), (64, 128, 256), (100, 1, 33), (129, 257, 65),
              (256, 256, 256), (300, 264, 520), (513, 72, 300), (1030, 130, 70)]


@pytest.mark.parametrize("pad", [0, 5, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,k,n", GRAD_SIZES)
def test_gradients(m, k, n, dtype, pad):
    gen = R.generator("grad", m, k, n, dtype, pad)
    name = ["gelu", "none", "relu", "silu"][(m + k + n + pad) % 4]
    x, w = R.rows(gen, m, k, dtype, pad), R.rows(gen, n, k, dtype, 0, k ** -0.5)
    dy, pre = R.rows(gen, m, n, dtype, pad), R.rows(gen, m, n, dtype, 0, 1.5)
    dx, dw, db = layer().tg_linear_grad(dy, x, w, pre=pre, act=name, bias_grad=True)
    want = R.linear_grads(dy, x, w, pre, name)
    for key, got in (("dx", dx), ("dw", dw), ("db", db)):
        R.within(got, *want[key], key)


@pytest.mark.parametrize("m,k,n", [(129, 121, 121), (57, 249, 313), (300, 505, 65), (1, 57, 1), (3, 1, 121)])
def test_gradients_of_odd_rows_inside_aligned_ones(m, k, n):
    """Rows start at 16-byte addresses and end inside a 4-byte word, the operands' last ones at the buffers' ends."""
    gen = R.generator("odd rows", m, k, n)

    def rows(a, b, std=1.0):
        ld = -(-b // 8) * 8
        flat = (torch.randn((a - 1) * ld + b, generator=gen) * std).to(BF16).cuda()
        return flat.as_strided((a, b), (ld, 1))

    x, w, dy, pre = rows(m, k), rows(n, k, k ** -0.5), rows(m, n), rows(m, n)
    for name in ("none", "silu"):
        dx, dw, db = layer().tg_linear_grad(dy, x, w, pre=pre, act=name, bias_grad=True)
        want = R.linear_grads(dy, x, w, pre, name)
        for key, got in (("dx", dx), ("dw", dw), ("db", db)):
            R.within(got, *want[key], key)
        want, z, bound = R.linear(x, w, None, name)
        R.within(layer().tg_linear(x, w, act=name), want, R.linear_bound(want, z, bound, BF16), "y")


@pytest.mark.parametrize("name", ["relu", "silu", "gelu"])
def test_gradients_against_differences(name):
    """Central differences of the loss sum(dy y) in 64 bits: their own error is h^2 / 6 times a third derivative (bounded by
    3 for these activations) times the fourth moment of the inputs, far below the bound."""
    gen = R.generator("differences", name)
    m, k, n, h = 5, 12, 9, 1e-4
    x, w = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16, std=k ** -0.5)
    bias, dy = R.rows(gen, 1, n, BF16)[0], R.rows(gen, m, n, BF16)
    _, pre = layer().tg_linear(x, w, bias=bias, act=name, keep_pre=True)
    dx, dw, db = layer().tg_linear_grad(dy, x, w, pre=pre, act=name, bias_grad=True)
    inputs = {"dx": R.f64(x), "dw": R.f64(w), "db": R.f64(bias)}
    g = R.f64(dy)

    def loss():
        return float((g * R.act(inputs["dx"] @ inputs["dw"].t() + inputs["db"], name)).sum())

    z = R.f64(inputs["dx"]) @ inputs["dw"].t() + inputs["db"]
    if name == "relu":  # differences hold away from the corner only
        assert (z.abs() > 10 * h).all()
    bounds = R.linear_grads(dy, x, w, z.to(BF16), name)
    for key, got in (("dx", dx), ("dw", dw), ("db", db)):
        t = inputs[key]
        # pre is rounded too: the slope moves by at most 0.8 times 2^-8 |z|
        dz = g.abs() * 0.8 * 2.0 ** -8 * z.abs() if name != "relu" else torch.zeros_like(g)
        extra = {"dx": dz @ inputs["dw"].abs(), "dw": dz.t() @ inputs["dx"].abs(), "db": dz.sum(0)}[key]
        for i in range(0, t.numel(), 3):
            flat = t.reshape(-1)
            keep = float(flat[i])
            flat[i] = keep + h
            up = loss()
            flat[i] = keep - h
            down = loss()
            flat[i] = keep
            far = abs((up - down) / (2 * h) - float(got.reshape(-1)[i]))
            assert far <= float((bounds[key][1] + 2 * extra).reshape(-1)[i]) + 1e-6, (key, i, far)


@pytest.mark.parametrize("m,k,n", [(0, 8, 8), (4, 0, 8), (4, 8, 0), (300, 0, 300)])
def test_empty_sizes(m, k, n):
    L = layer()
    x, w = torch.ones(m, k, device="cuda", dtype=BF16), torch.ones(n, k, device="cuda", dtype=BF16)
    bias, dy = torch.full((n,), 2.0, device="cuda", dtype=BF16), torch.ones(m, n, device="cuda", dtype=BF16)
    y, pre = L.tg_linear(x, w, bias=bias, act="relu", keep_pre=True)
    assert y.shape == (m, n) and bool((y == 2 + k).all())
    dx, dw, db = L.tg_linear_grad(dy, x, w, pre=pre, act="relu", bias_grad=True)
    assert bool((dx == n).all()) and bool((dw == m).all()) and bool((db == m).all())


def test_residual_in_place_and_given_workspace():
    L = layer()
    gen = R.generator("in place")
    x, w, r = R.rows(gen, 130, 256, BF16), R.rows(gen, 264, 256, BF16, std=1 / 16), R.rows(gen, 130, 264, BF16)
    want = L.tg_linear(x, w, residual=r)
    got = L.tg_linear(x, w, residual=r, out=r, workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    assert got is r and torch.equal(got, want)


def test_repeatable_and_on_another_stream():
    L = layer()
    gen = R.generator("stream")
    x, w, dy = R.rows(gen, 500, 1100, BF16), R.rows(gen, 700, 1100, BF16, std=1 / 32), R.rows(gen, 500, 700, BF16)
    first = [L.tg_linear(x, w)] + list(L.tg_linear_grad(dy, x, w, bias_grad=True))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [L.tg_linear(x, w)] + list(L.tg_linear_grad(dy, x, w, bias_grad=True))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("m", [1, 40, 300])
def test_nan_and_infinity_stay_in_their_rows_and_columns(m):
    """Bytes past a row's end must not reach a result: what lies there is NaN."""
    L = layer()
    gen = R.generator("nan", m)
    for k, pad in ((72, 8), (70, 10), (69, 3), (64, 64)):
        x, w = R.rows(gen, m, k, BF16, pad), R.rows(gen, 90, k, BF16, pad)
        for t in (x, w):
            t.as_strided((t.shape[0] - 1, pad), t.stride(), t.storage_offset() + k).fill_(float("nan"))
        y = L.tg_linear(x, w)
        assert bool(torch.isfinite(y).all())
        x[m // 2, k - 1] = float("inf")
        w[3, 0] = float("nan")
        y = L.tg_linear(x, w)
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        want[m // 2], want[:, 3] = True, True
        assert torch.equal(bad, want)
        dy = R.rows(gen, m, 90, BF16, 6)
        dy.as_strided((m - 1, 6), dy.stride(), dy.storage_offset() + 90).fill_(float("nan"))
        w[3, 0] = 1.0
        x[m // 2, k - 1] = 1.0
        dx, dw, db = L.tg_linear_grad(dy, x, w, bias_grad=True)
        assert all(bool(torch.isfinite(t).all()) for t in (dx, dw, db))


def test_rows_further_apart_than_32_bits_reach():
    L = layer()
    gen = R.generator("far")
    m, k, n, ld = 3, 72, 40, 1 << 30
    small, w = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16)
    far = torch.empty(2 * ld + 128, dtype=BF16, device="cuda")
    x = far.as_strided((m, k), (ld, 1))
    x.copy_(small)
    out = far.as_strided((m, n), (ld, 1), 128 - n)
    assert torch.equal(L.tg_linear(x, w), L.tg_linear(small, w))
    want = L.tg_linear(small, w, act="silu")
    assert torch.equal(L.tg_linear(x, w, act="silu", out=out), want)
    dy = R.rows(gen, m, n, BF16)
    for a, b in zip(L.tg_linear_grad(dy, x, w), L.tg_linear_grad(dy, small, w)):
        assert a is b or torch.equal(a, b)


def test_graph_replays():
    L = layer()
    gen = R.generator("graph")
    x, w, dy = R.rows(gen, 200, 512, BF16), R.rows(gen, 320, 512, BF16, std=1 / 16), R.rows(gen, 200, 320, BF16)

    def step():
        y, pre = L.tg_linear(x, w, act="gelu", keep_pre=True)
        return (y, *L.tg_linear_grad(dy, x, w, pre=pre, act="gelu", bias_grad=True))

    step()
    torch.cuda.synchronize()
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
    bad = [lambda: L.tg_linear(x.float(), w), lambda: L.tg_linear(x, w.half()), lambda: L.tg_linear(x, w[:, :7]),
           lambda: L.tg_linear(x.t(), w), lambda: L.tg_linear(x[0], w), lambda: L.tg_linear(x.cpu(), w),
           lambda: L.tg_linear(x, w, act="tanh"), lambda: L.tg_linear(x, w, bias=x[0]),
           lambda: L.tg_linear(x, w, residual=x), lambda: L.tg_linear(x, w, out_dtype=torch.float16),
           lambda: L.tg_linear(x, w, x_scale=torch.ones(4, device="cuda"), w_scale=torch.ones(6, device="cuda")),
           lambda: L.tg_linear(x[:1].expand(4, 8), w), lambda: L.tg_linear(x, w, out=torch.zeros(4, 6, device="cuda")),
           lambda: L.tg_linear_grad(x, x, w), lambda: L.tg_linear_grad(torch.zeros(4, 6, device="cuda", dtype=BF16), x, w, act="gelu")]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {k} was taken")
    from paper_2606_16907_amd.tangram import TangramError
    dy = torch.zeros(4, 6, device="cuda", dtype=BF16)
    with pytest.raises(TangramError, match="workspace"):
        L.tg_linear_grad(dy, x, w, pre=dy, act="relu", workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
