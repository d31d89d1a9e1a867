"""The layer norm and its gradient against 64 bits."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E4M3, E32, TINY, U

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def sums(cols):
    """A sum of n terms of any signs is off by at most this times the sum of their sizes: the kernels add at most n / 64 of
    them, and 24 more, in a row."""
    return (cols / 64 + 24) * E32


def norm(x, w, b, r):
    h = R.f64(x) if r is None else R.f64(x) + R.f64(r)
    mean = h.mean(1, keepdim=True)
    rstd = 1 / ((h - mean).square().mean(1, keepdim=True) + EPS).sqrt()
    return h, mean, rstd, (h - mean) * rstd * R.f64(w) + (0 if b is None else R.f64(b))


def stats_bounds(h, mean, rstd, size, cols):
    """(mean's, rstd's relative): the first sum's mean m1 is off by sums(n) mean|h| =: d; the second sum, of h - m1, takes d
    out again up to its own rounding, sums(n) (mean|h - mean| + d) and e of |h|.  The deviations are each off by that and e of
    |h|, so their squares by twice their product."""
    d = sums(cols) * h.abs().mean(1, keepdim=True)
    dev = (h - mean).abs().mean(1, keepdim=True)
    bm = sums(cols) * (dev + 2 * d) + 4 * E32 * size.amax(1, keepdim=True)
    off = bm + 4 * E32 * size.amax(1, keepdim=True) + d
    br = (sums(cols) + 12 * E32) + rstd.square() * (2 * dev * off + 4 * off.square())
    return bm, br


SHAPES = [(1, 1), (1, 8192), (2, 3), (3, 7), (5, 8), (4, 64), (9, 100), (6, 511), (3, 512), (7, 513), (2, 1024), (5, 1030), (3, 2048), (300, 2056),
          (3, 4096), (261, 4099), (3, 4999), (2, 8192), (258, 8192), (2, 8200), (260, 6152), (3, 12288), (259, 12290), (3, 16384), (2, 16390), (2, 33000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad", [0, 5])
def test_forward(rows, cols, dtype, pad):
    gen = R.generator("ln", rows, cols, dtype, pad)
    x, w = R.rows(gen, rows, cols, dtype, pad), R.rows(gen, 1, cols, dtype)[0]
    b = R.rows(gen, 1, cols, dtype)[0] if cols % 2 or pad else None
    r = (R.rows(gen, rows, cols, dtype, pad, 3.0) + 2.0) if (rows + cols) % 2 or pad else None
    f = layer().tg_layer_norm(x, w, bias=b, residual=r, eps=EPS)
    h, mean, rstd, y = norm(x, w, b, r)
    size = h.abs() if r is None else R.f64(x).abs() + R.f64(r).abs()
    bm, br = stats_bounds(h, mean, rstd, size, cols)
    R.within(f.mean, mean[:, 0], bm[:, 0], "mean")
    R.within(f.rstd, rstd[:, 0], br[:, 0] * rstd[:, 0], "rstd")
    scaled = ((h - mean) * rstd * R.f64(w)).abs()
    slack = (bm + 4 * E32 * size) * rstd * R.f64(w).abs() + (br + 8 * E32) * scaled + 4 * E32 * (scaled + y.abs())
    R.within(f.y, y, 1.01 * U[dtype] * y.abs() + 1.01 * slack + TINY[dtype], "y")
    if r is None:
        assert f.hidden is x
    else:
        R.within(f.hidden, h, 1.01 * U[dtype] * h.abs() + 2 * E32 * size + TINY[dtype], "hidden")


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_forward_in_8_bits(rows, cols, dtype):
    gen = R.generator("ln e4m3", rows, cols, dtype)
    x, w, r = R.rows(gen, rows, cols, dtype, 3), R.rows(gen, 1, cols, dtype)[0], R.rows(gen, rows, cols, dtype)
    b = R.rows(gen, 1, cols, dtype)[0]
    f = layer().tg_layer_norm(x, w, bias=b, residual=r, eps=EPS, out_dtype=E4M3)
    assert f.mean is None and f.rstd is None
    h, mean, rstd, y = norm(x, w, b, r)
    size = R.f64(x).abs() + R.f64(r).abs()
    bm, br = stats_bounds(h, mean, rstd, size, cols)
    scaled = ((h - mean) * rstd * R.f64(w)).abs()
    slack = 1.01 * ((bm + 4 * E32 * size) * rstd * R.f64(w).abs() + (br + 8 * E32) * scaled + 4 * E32 * (scaled + y.abs()))
    most = y.abs().amax(1)
    R.within(f.scale, most / 448, 4 * E32 * most / 448 + slack.amax(1) / 448, "scale")
    got = R.f64(f.y.float()) * R.f64(f.scale)[:, None]
    R.within(got, y, (2.0 ** -4 * 1.001) * y.abs() + 2.0 ** -10 * 1.001 * R.f64(f.scale)[:, None] + 2 * slack, "y")
    assert float(f.y.float().abs().max()) <= 448.0


@pytest.mark.parametrize("rows,cols", SHAPES + [(0, 40), (700, 72), (1030, 513), (1100, 40), (64, 500), (65, 500), (1, 33000), (0, 33000), (2, 5000)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad", [0, 5])
def test_gradients(rows, cols, dtype, pad):
    gen = R.generator("ln grad", rows, cols, dtype, pad)
    hid, w = R.rows(gen, rows, cols, dtype, pad), (1 + R.rows(gen, 1, cols, F32)[0] * 0.2).to(dtype)
    dy = R.rows(gen, rows, cols, dtype, pad)
    dh = R.rows(gen, rows, cols, dtype, pad) if (rows + cols) % 2 else None
    h = R.f64(hid)
    m = h.mean(1, keepdim=True)
    m32, s32 = m[:, 0].float().cuda(), (1 / ((h - m).square().mean(1) + EPS).sqrt()).float().cuda()
    dx, dw, db = layer().tg_layer_norm_grad(dy, hid, w, m32, s32, dhidden=dh)
    m, s = R.f64(m32)[:, None], R.f64(s32)[:, None]
    g, xhat = R.f64(dy) * R.f64(w), (h - m) * s
    ex = 4 * E32 * (xhat.abs() + s * (h.abs() + m.abs()))  # xhat's own error
    first, second = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    b1 = sums(cols) * g.abs().mean(1, keepdim=True) + 4 * E32 * first.abs()
    b2 = sums(cols) * (g * xhat).abs().mean(1, keepdim=True) + (g.abs() * ex).mean(1, keepdim=True) + 4 * E32 * second.abs()
    want = s * (g - first - xhat * second) + (0 if dh is None else R.f64(dh))
    err = s * (b1 + xhat.abs() * b2 + ex * second.abs() + 8 * E32 * (g.abs() + first.abs() + (xhat * second).abs())) + 8 * E32 * want.abs()
    R.within(dx, want, 1.01 * U[dtype] * want.abs() + 2 * err + TINY[dtype], "dx")
    term = R.f64(dy) * xhat
    R.within(dw, term.sum(0), 1.01 * U[dtype] * term.sum(0).abs() + (rows + 16) * E32 * term.abs().sum(0) + (R.f64(dy).abs() * ex).sum(0) + TINY[dtype], "dweight")
    d = R.f64(dy)
    R.within(db, d.sum(0), 1.01 * U[dtype] * d.sum(0).abs() + (rows + 16) * E32 * d.abs().sum(0) + TINY[dtype], "dbias")
    dx2, dw2, none = layer().tg_layer_norm_grad(dy, hid, w, m32, s32, dhidden=dh, bias_grad=False)
    assert none is None and torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cols", [8, 520, 1032, 1544, 2056, 4104, 8200, 12296])
def test_gradients_at_every_end_of_a_row(cols, dtype):
    """Last units of 1 to 7 elements, in each width that a kernel is made for; dx may be dy or dhidden there, too."""
    for end in range(1, 8):
        rows = 19 + end
        test_gradients(rows, cols + end, dtype, 5)
        gen = R.generator("ln ends", cols, end, dtype)
        hid, w, dy, dh = (R.rows(gen, n, cols + end, dtype, 3) for n in (rows, 1, rows, rows))
        stats = hid.float().mean(1), 1 / hid.float().std(1)
        want = layer().tg_layer_norm_grad(dy, hid, w[0], *stats, dhidden=dh)
        for place in (dy.clone(), dh.clone()):
            other = {"dhidden": place} if torch.equal(place, dh) else {"dhidden": dh}
            got = layer().tg_layer_norm_grad(dy if torch.equal(place, dh) else place, hid, w[0], *stats, dx=place, **other)
            assert all(torch.equal(a, b) for a, b in zip(got, want, strict=True))


def test_gradient_against_differences():
    gen = R.generator("ln differences")
    rows, cols, step = 3, 37, 1e-5
    x, w, b, dy = R.rows(gen, rows, cols, F32), R.rows(gen, 1, cols, F32)[0], R.rows(gen, 1, cols, F32)[0], R.rows(gen, rows, cols, F32)
    f = layer().tg_layer_norm(x, w, bias=b, eps=EPS)
    dx, dw, db = layer().tg_layer_norm_grad(dy, f.hidden, w, f.mean, f.rstd)
    at = {"x": R.f64(x), "w": R.f64(w), "b": R.f64(b)}

    def loss():
        d = at["x"] - at["x"].mean(1, keepdim=True)
        return float((R.f64(dy) * (d / (d.square().mean(1, keepdim=True) + EPS).sqrt() * at["w"] + at["b"])).sum())

    for key, got in (("x", dx), ("w", dw), ("b", db)):
        flat = at[key].reshape(-1)
        for i in range(0, flat.numel(), 5):
            keep = float(flat[i])
            flat[i] = keep + step
            up = loss()
            flat[i] = keep - step
            down = loss()
            flat[i] = keep
            # the third derivative is of order 1, rounding of the loss about 1e-15 / step
            assert abs((up - down) / (2 * step) - float(got.reshape(-1)[i])) <= 2e-5, (key, i)


@pytest.mark.parametrize("cols", [100, 700, 1025, 5000, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_rows_far_from_zero(cols, dtype):
    """A constant row has deviations of 0, and one of small steps around 1000 keeps them (the steps are whole in 16 bits)."""
    L = layer()
    x = torch.full((2, cols), 1000.0, device="cuda", dtype=dtype)
    x[1] += 8.0 * (torch.arange(cols, device="cuda") % 3 - 1).to(dtype)
    w = torch.ones(cols, device="cuda", dtype=dtype)
    f = L.tg_layer_norm(x, w, eps=EPS)
    assert bool((f.y[0] == 0).all()) and float(f.mean[0]) == 1000.0
    h = R.f64(x)
    y = (h - h.mean(1, keepdim=True)) / (h.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
    # a mean off by 2 units of 1000 in 32 bits moves the steps of 8 by 2^-13 of 8
    R.within(f.y[1:], y[1:], 1.01 * U[dtype] * y[1:].abs() + 2.0 ** -13, "y")


def test_zero_rows_and_rows_that_are_not_finite():
    L = layer()
    x = torch.ones(6, 700, device="cuda", dtype=BF16)
    x[:, ::2] = -1
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 699] = float("inf")
    w, b = torch.ones(700, device="cuda", dtype=BF16), torch.full((700,), 0.5, device="cuda", dtype=BF16)
    y = L.tg_layer_norm(x, w, bias=b).y
    assert bool((y[1] == 0.5).all()) and bool(torch.isnan(y[[2, 3]]).all()) and bool(torch.isfinite(y[[0, 4, 5]]).all())
    f = L.tg_layer_norm(x, w, out_dtype=E4M3)
    q = f.y.float()
    assert float(f.scale[1]) == 1.0 and bool((q[1] == 0).all()) and bool(torch.isnan(q[[2, 3]]).all())
    assert f.scale[[2, 3]].tolist() == [1.0, 1.0] and bool((q[[0, 4, 5]].abs() == 448).all())


def test_empty_rows_and_no_columns():
    L = layer()
    w = torch.ones(40, device="cuda")
    f = L.tg_layer_norm(torch.ones(0, 40, device="cuda"), w)
    assert f.y.shape == (0, 40)
    dx, dw, db = L.tg_layer_norm_grad(f.y, f.hidden, w, f.mean, f.rstd)
    assert dx.shape == (0, 40) and bool((dw == 0).all()) and bool((db == 0).all())
    f = L.tg_layer_norm(torch.ones(3, 0, device="cuda"), w[:0])
    assert f.y.shape == (3, 0) and f.rstd.shape == (3,)


def test_rows_further_apart_than_32_bits_reach():
    L = layer()
    gen = R.generator("ln far")
    ld = 1 << 31
    small, w = R.rows(gen, 3, 300, BF16), R.rows(gen, 1, 300, BF16)[0]
    far = torch.empty(2 * ld + 300, dtype=BF16, device="cuda").as_strided((3, 300), (ld, 1))
    far.copy_(small)
    a, b = L.tg_layer_norm(far, w, bias=w), L.tg_layer_norm(small, w, bias=w)
    assert torch.equal(a.y, b.y)
    for p, q in zip(L.tg_layer_norm_grad(far, far, w, a.mean, a.rstd), L.tg_layer_norm_grad(small, small, w, b.mean, b.rstd)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("rows,cols", [(700, 1000), (3, 40000)])
def test_outputs_in_the_place_of_inputs(rows, cols):
    L, gen = layer(), R.generator("ln places", rows, cols)
    x, w, dy, dh = R.rows(gen, rows, cols, BF16), R.rows(gen, 1, cols, BF16)[0], R.rows(gen, rows, cols, BF16), R.rows(gen, rows, cols, BF16)
    f = L.tg_layer_norm(x, w)
    want = L.tg_layer_norm_grad(dy, x, w, f.mean, f.rstd, dhidden=dh)
    for place in (0, 1):
        a, b = dy.clone(), dh.clone()
        got = L.tg_layer_norm_grad(a, x, w, f.mean, f.rstd, dhidden=b, dx=(a, b)[place])
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("rows,cols", [(70, 1000), (3, 40000), (300, 12288)])
@pytest.mark.parametrize("place", ["x", "residual"])
def test_hidden_in_the_place_of_an_input(rows, cols, place):
    """Through the C entry, which allows it."""
    import ctypes
    L, gen = layer(), R.generator("ln hidden", rows, cols)
    x, r, w = R.rows(gen, rows, cols, BF16), R.rows(gen, rows, cols, BF16), R.rows(gen, 1, cols, BF16)[0]
    want = L.tg_layer_norm(x, w, residual=r)
    y, hidden = torch.empty_like(x), x if place == "x" else r
    a = L.TgLayerNormArgs(x.data_ptr(), r.data_ptr(), w.data_ptr(), None, hidden.data_ptr(), y.data_ptr(), None, None, None, rows, cols, cols, cols, cols,
                          cols, EPS, 1, 1, 0)
    assert L.load_library().tg_layer_norm(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(y, want.y) and torch.equal(hidden, want.hidden)


def test_repeatable_and_replayed():
    L = layer()
    gen = R.generator("ln graph")
    x, w, r = R.rows(gen, 700, 1000, BF16), R.rows(gen, 1, 1000, BF16)[0], R.rows(gen, 700, 1000, BF16)

    def step():
        f = L.tg_layer_norm(x, w, bias=w, residual=r)
        return (f.y, f.hidden, f.mean, f.rstd, *L.tg_layer_norm_grad(x, f.hidden, w, f.mean, f.rstd, dhidden=r))

    first = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), k
        assert all(torch.equal(a, b) for a, b in zip(out, first)) or k
        x.copy_(R.rows(gen, 700, 1000, BF16))


def test_refusals():
    L = layer()
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    s = torch.ones(4, device="cuda")
    bad = [lambda: L.tg_layer_norm(x.double(), w), lambda: L.tg_layer_norm(x, w[:7]), lambda: L.tg_layer_norm(x, w, bias=w.half()),
           lambda: L.tg_layer_norm(x, w, out_dtype=torch.float16), lambda: L.tg_layer_norm(x, w, residual=x[:2]),
           lambda: L.tg_layer_norm(x.t(), w[:4]), lambda: L.tg_layer_norm(x.cpu(), w),
           lambda: L.tg_layer_norm_grad(x, x, w, w, s), lambda: L.tg_layer_norm_grad(x, x, w, s, s, dbias=s)]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {k} was taken")
    from paper_2606_16907_amd.tangram import TangramError
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(TangramError, match="eps"):
            L.tg_layer_norm(x, w, eps=eps)
