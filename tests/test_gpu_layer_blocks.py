"""The quantiser and the 8-bit product with a scale for every block of 128, against 64 bits."""
import pytest
import torch

from tests import layer_ref as R
from tests.gated_ref import dropped
from tests.layer_ref import E4M3, E32

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E8M0 = torch.float8_e8m0fnu
BLOCK = 128


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def values(scale):
    """A scale's values in 64 bits."""
    t = scale.cpu()
    if t.dtype == E8M0:
        code = t.view(torch.uint8).to(torch.float64)
        return torch.where(code == 255, torch.full_like(code, float("nan")), torch.exp2(code - 127))
    return t.to(torch.float64)


def spread(scale, rows, cols, block_rows):
    t = values(scale).repeat_interleave(BLOCK, 1)[:, :cols]
    return t.repeat_interleave(block_rows, 0)[:rows]


def wanted_scale(x, block_rows, powers):
    """From x in 64 bits."""
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // BLOCK)
    a = torch.zeros(nr * block_rows, nc * BLOCK, dtype=torch.float64)
    a[:rows, :cols] = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    most = a.view(nr, block_rows, nc, BLOCK).amax((1, 3))
    s = (most.float() / 448).clamp_min(2.0 ** -126).to(torch.float64)
    if powers:
        part, e = torch.frexp(s)
        s = torch.ldexp(torch.ones_like(s), torch.where(part == 0.5, e - 1, e))
    return torch.where(most > 0, s, torch.ones_like(s))


QUANTIZE_SIZES = [(1, 1), (1, 127), (2, 128), (3, 129), (5, 64), (4, 1000), (7, 2048), (3, 2056), (2, 8199), (130, 300), (129, 513), (257, 128), (1, 40000)]


@pytest.mark.parametrize("rows,cols", QUANTIZE_SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("powers", [False, True])
def test_quantize(rows, cols, dtype, block_rows, powers):
    gen = R.generator("quantize", rows, cols, dtype, block_rows, powers)
    pad = (rows + cols) % 3
    size = torch.randn(cols, generator=gen).mul(2).exp().cuda()
    x = (R.rows(gen, rows, cols, F32, pad) * size).to(dtype)
    q = layer().tg_quantize(x, block_rows=block_rows, scale_dtype=E8M0 if powers else F32)
    want = R.f64(x)
    s = wanted_scale(want, block_rows, powers)
    assert q.scale.shape == s.shape
    if powers:
        assert torch.equal(values(q.scale), s)
    else:
        R.within(q.scale, s, E32 * s, "scale")
    # half a step of the type: 2^-4 of the value, 2^-10 of the scale below 2^-6; the quotient is rounded to 32 bits before
    at = spread(q.scale, rows, cols, block_rows)
    R.within(R.f64(q.y.float()) * at, want, 2.0 ** -4 * (1 + 2 ** -18) * want.abs() + 2.0 ** -10 * (1 + 2 ** -18) * at, "y")
    # the quotient is the nearest 32-bit number: codes are those of the division but beside a border between two
    exact = (want / at).to(F32)
    assert float(((exact.to(E4M3).float()) != q.y.float().cpu()).float().mean()) <= 1e-5


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("powers", [False, True])
def test_quantize_numbers_at_the_ends(block_rows, powers):
    L, kind = layer(), E8M0 if powers else F32
    x = torch.zeros(128, 7 * 128, device="cuda")
    x[:, 128:256] = 1e-40                       # subnormal
    x[:, 256:384] = 3e38
    x[3, 384 + 5], x[4, 384 + 6] = float("nan"), 7.0
    x[3, 512 + 5], x[4, 512 + 6] = float("inf"), -7.0
    x[3, 640] = 448.0
    x[:, 768:] = 2.0 ** -120
    q = L.tg_quantize(x, block_rows=block_rows, scale_dtype=kind)
    y, s = q.y.float().cpu(), values(q.scale)
    assert bool((y[:, :128] == 0).all()) and bool((s[:, 0] == 1).all())
    assert bool((s[:, 1] == 2.0 ** -126).all())
    assert bool(((y[:, 128:256].double() * 2.0 ** -126 - 1e-40).abs() <= 2.0 ** -136).all())
    assert bool(torch.isfinite(s).all()) and bool((y[:, 256:384].abs() <= 448).all())
    assert torch.isnan(y).nonzero().tolist() == [[3, 384 + 5], [3, 512 + 5]]
    row = 0 if block_rows == 128 else 4
    assert float(s[row, 3]) >= 7 / 448 * 0.999999 and float(y[4, 384 + 6]) * float(s[row, 3]) == pytest.approx(7, rel=2 ** -4)
    assert float(y[4, 512 + 6]) * float(s[row, 4]) == pytest.approx(-7, rel=2 ** -4)
    assert float(y[3, 640]) == 448 and float(s[0 if block_rows == 128 else 3, 5]) == 1
    assert bool(((y[:, 768:] * s[0, 6] - 2.0 ** -120).abs() <= 2.0 ** -124).all())


def test_quantize_given_places_and_nothing_past_them():
    L, gen = layer(), R.generator("places")
    x = R.rows(gen, 70, 300, BF16, 5)
    out = torch.full((71, 320), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.full((71, 8), 5.0, device="cuda")
    q = L.tg_quantize(x, out=out.view(E4M3)[:70, :300], scale=scale[:70, :3])
    r = L.tg_quantize(x.contiguous())
    assert torch.equal(q.y.view(torch.uint8), r.y.view(torch.uint8)) and torch.equal(q.scale, r.scale)
    assert bool((out[70] == 0x55).all()) and bool((out[:, 300:] == 0x55).all()) and bool((scale[70] == 5).all()) and bool((scale[:, 3:] == 5).all())
    assert L.tg_quantize(x[:0]).y.shape == (0, 300) and L.tg_quantize(x[:, :0]).scale.shape == (70, 0)


def operands(gen, m, k, n, powers, pad=0):
    """8-bit x and w with scales of their own, within rows that are wider, the pad NaN."""
    def one(rows, block_rows, std):
        bits = torch.randint(0, 127, (rows, k + pad), generator=gen, dtype=torch.uint8) | (torch.randint(0, 2, (rows, k + pad), generator=gen, dtype=torch.uint8) << 7)
        small = torch.rand(rows, k + pad, generator=gen) < 0.5
        bits = torch.where(small, bits & 0x9f, bits).cuda()
        bits[:, k:] = 0x7f
        shape = (-(-rows // block_rows), -(-k // BLOCK) + pad)
        scale = torch.randn(shape, generator=gen).mul(1.0).exp().mul(std / 100)
        scale = torch.randint(110, 126, shape, generator=gen, dtype=torch.uint8).view(E8M0) if powers else scale
        scale = scale.cuda()
        scale[:, -(-k // BLOCK):] = float("nan")
        return bits.view(E4M3)[:, :k], scale[:, :-(-k // BLOCK)]
    return (*one(m, 1, 1.0), *one(n, BLOCK, k ** -0.5))


def block_linear(x, xs, w, ws):
    """(z, bound): blocks' sums of any order in the matrix instruction, then one product and one addition a block."""
    a = R.f64(x.float()) * spread(xs, *x.shape, 1)
    b = R.f64(w.float()) * spread(ws, *w.shape, BLOCK)
    z, size = a @ b.t(), a.abs() @ b.abs().t()
    blocks = -(-x.shape[1] // BLOCK)
    return z, dropped(a, b) + (BLOCK + blocks + 16) * E32 * size


def check(m, k, n, powers, pad, act="none", bias=False, residual=False, out=BF16):
    gen = R.generator("blocks", m, k, n, powers, pad)
    x, xs, w, ws = operands(gen, m, k, n, powers, pad)
    b = R.rows(gen, 1, n, out)[0] if bias else None
    r = R.rows(gen, m, n, out, pad) if residual else None
    y = layer().tg_block_linear(x, w, xs, ws, bias=b, act=act, residual=r, out_dtype=out)
    z, bound = block_linear(x, xs, w, ws)
    if bias:
        z, bound = z + R.f64(b), bound + 4 * E32 * R.f64(b).abs()
    want = R.act(z, act) + (R.f64(r) if residual else 0)
    R.within(y, want, R.linear_bound(want, z, bound, out, r), "y")


@pytest.mark.parametrize("powers", [False, True])
@pytest.mark.parametrize("pad", [0, 3, 16])
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 128, 16), (1, 4096, 130), (3, 129, 17), (8, 640, 257), (9, 256, 128), (16, 1000, 129), (33, 127, 300),
                                   (64, 2048, 100), (17, 4096, 8300), (40, 8200, 520), (65, 513, 129), (128, 128, 128), (130, 1152, 255), (257, 300, 520), (300, 4096, 136), (600, 1040, 1030)])
def test_block_linear(m, k, n, powers, pad):
    check(m, k, n, powers, pad, act=["none", "relu", "silu", "gelu"][(m + n) % 4], bias=bool(k % 2), residual=bool(m % 2), out=[BF16, F16][n % 2])


@pytest.mark.parametrize("powers", [False, True])
@pytest.mark.parametrize("m,k,n,pad", [(1, 14336, 1024, 0), (4, 20483, 33, 5), (1500, 8200, 3000, 8), (3500, 2064, 4075, 0), (3841, 1999, 3841, 3), (3000, 16400, 1500, 0), (4352, 4100, 4352, 0)])
def test_shared_sums_and_large_tiles(m, k, n, pad, powers):
    check(m, k, n, powers, pad, residual=True)


def test_quantised_operands_multiply_to_the_product():
    """The two operators together, against the product of the values before they are quantised: each value is off by at most
    2^-4 of itself or 2^-10 of its block's scale, independently of the others (8 standard deviations, 1 / sqrt(3) of that)."""
    L, gen = layer(), R.generator("together")
    m, k, n = 200, 1500, 300
    x, w = R.rows(gen, m, k, BF16), R.rows(gen, n, k, BF16, std=k ** -0.5)
    for kind in (F32, E8M0):
        qx, qw = L.tg_quantize(x, scale_dtype=kind), L.tg_quantize(w, block_rows=128, scale_dtype=kind)
        y = L.tg_block_linear(qx.y, qw.y, qx.scale, qw.scale)
        a, b = R.f64(x), R.f64(w)
        ea = 2.0 ** -4 * a.abs() + 2.0 ** -10 * spread(qx.scale, m, k, 1)
        eb = 2.0 ** -4 * b.abs() + 2.0 ** -10 * spread(qw.scale, n, k, 128)
        spreads = (ea.square() @ b.square().t() + a.square() @ eb.square().t() + ea.square() @ eb.square().t()).sqrt() / 3 ** 0.5
        want = a @ b.t()
        R.within(y, want, 8 * spreads + 2.0 ** -8 * want.abs() + 1.2 * dropped(a, b) + 300 * E32 * (a.abs() @ b.abs().t()), "y")


@pytest.mark.parametrize("powers", [False, True])
@pytest.mark.parametrize("m", [1, 8, 40, 300])
def test_nan_stays_in_its_rows_and_columns(m, powers):
    L, gen = layer(), R.generator("block nan", m, powers)
    for k, pad in ((160, 16), (159, 3), (128, 0)):
        x, xs, w, ws = operands(gen, m, k, 300, powers, pad)
        assert bool(torch.isfinite(L.tg_block_linear(x, w, xs, ws)).all())
        x.view(torch.uint8)[m // 2, k - 1] = 0x7f
        w.view(torch.uint8)[3, 0] = 0xff
        ws[2, 0] = float("nan")
        if m > 2:
            xs[0, -1] = float("nan")
        bad = torch.isnan(L.tg_block_linear(x, w, xs, ws))
        want = torch.zeros_like(bad)
        want[m // 2], want[:, 3], want[:, 256:] = True, True, True
        if m > 2:
            want[0] = True
        assert torch.equal(bad, want)


@pytest.mark.parametrize("m,k,n", [(0, 128, 8), (4, 0, 8), (4, 128, 0), (300, 0, 300)])
def test_empty_sizes(m, k, n):
    L = layer()
    x, w = (torch.zeros(s, dtype=torch.uint8, device="cuda").view(E4M3) for s in ((m, k), (n, k)))
    xs, ws = torch.ones(m, k // 128, device="cuda"), torch.ones(-(-n // 128), k // 128, device="cuda")
    bias = torch.full((n,), 3.0, device="cuda", dtype=BF16)
    assert bool((L.tg_block_linear(x, w, xs, ws, bias=bias, act="relu") == 3).all())


def test_residual_in_place_repeatable_replayed_and_on_another_stream():
    L, gen = layer(), R.generator("block graph")
    m, k, n = 200, 640, 320
    x, r = R.rows(gen, m, k, BF16), R.rows(gen, m, n, BF16)
    w = L.tg_quantize(R.rows(gen, n, k, BF16, std=k ** -0.5), block_rows=128)

    def step():
        q = L.tg_quantize(x)
        return L.tg_block_linear(q.y, w.y, q.scale, w.scale, residual=r), L.tg_block_linear(q.y[:1], w.y, q.scale[:1], w.scale, residual=r[:1])

    first = step()
    again = r.clone()
    q = L.tg_quantize(x)
    assert L.tg_block_linear(q.y, w.y, q.scale, w.scale, residual=again, out=again) is again and torch.equal(again, first[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(3):
        x.copy_(R.rows(gen, m, k, BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), turn


def test_rows_further_apart_than_32_bits_reach():
    L, gen = layer(), R.generator("block far")
    m, k, n, ld = 3, 160, 40, 1 << 31
    small = R.rows(gen, m, k, F32).to(E4M3)
    w = L.tg_quantize(R.rows(gen, n, k, BF16), block_rows=128)
    xs = torch.rand(m, 2, generator=gen).cuda()
    far = torch.zeros(2 * ld + 256, dtype=torch.uint8, device="cuda").view(E4M3)
    x = far.as_strided((m, k), (ld, 1))
    x.copy_(small)
    assert torch.equal(L.tg_block_linear(x, w.y, xs, w.scale), L.tg_block_linear(small, w.y, xs, w.scale))
    wide = far.view(torch.uint8)[: (ld // 2) * 4].view(BF16)
    rows = wide.as_strided((2, k), (1 << 30, 1))
    rows.copy_(R.rows(gen, 2, k, BF16))
    a, b = L.tg_quantize(rows), L.tg_quantize(rows.contiguous())
    assert torch.equal(a.scale, b.scale) and torch.equal(a.y.view(torch.uint8), b.y.view(torch.uint8))


def test_refusals():
    L = layer()
    x, w = (torch.zeros(s, dtype=torch.uint8, device="cuda").view(E4M3) for s in ((4, 256), (130, 256)))
    xs, ws = torch.ones(4, 2, device="cuda"), torch.ones(2, 2, device="cuda")
    f = torch.zeros(4, 256, device="cuda")
    bad = [lambda: L.tg_block_linear(f, w, xs, ws), lambda: L.tg_block_linear(x, w[:, :100], xs, ws), lambda: L.tg_block_linear(x, w, xs[:3], ws),
           lambda: L.tg_block_linear(x, w, xs, ws[:1]), lambda: L.tg_block_linear(x, w, xs, ws.to(E8M0)), lambda: L.tg_block_linear(x, w, xs.half(), ws.half()),
           lambda: L.tg_block_linear(x, w, xs, ws, out_dtype=F32), lambda: L.tg_block_linear(x, w, xs, ws, bias=xs[0]),
           lambda: L.tg_block_linear(x, w, xs, ws, act="tanh"), lambda: L.tg_block_linear(x, w, xs.t().contiguous().t(), ws),
           lambda: L.tg_quantize(x), lambda: L.tg_quantize(f, block_rows=64), lambda: L.tg_quantize(f, scale_dtype=F16), lambda: L.tg_quantize(f.cpu()),
           lambda: L.tg_quantize(f.t()), lambda: L.tg_quantize(f, out=f), lambda: L.tg_quantize(f, scale=xs[:3])]
    for k, g in enumerate(bad):
        with pytest.raises(ValueError):
            g()
            pytest.fail(f"call {k} was taken")
    from paper_2606_16907_amd.tangram import TangramError
    far = torch.ones(2 * (1 << 21) * 4, device="cuda").as_strided((4, 2), (1 << 21, 1))
    with pytest.raises(TangramError, match="row stride"):
        L.tg_block_linear(x, w, far, ws)
