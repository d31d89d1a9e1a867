"""The root-mean-square norm and its gradient against 64 bits."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E4M3, E32, TINY, U

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-6


def layer():
    from paper_2606_16907_amd import layer as L
    return L


def norm(x, w, r):
    h = R.f64(x) if r is None else R.f64(x) + R.f64(r)
    rstd = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    return h, rstd, h * rstd * R.f64(w)


# a sum of n squares, each of them positive, is off by at most n/T + log steps of 32 bits: (n / 64 + 24) e covers every split
def stat_error(cols):
    return (cols / 64 + 24) * E32


SHAPES = [(1, 1), (1, 8192), (2, 3), (3, 7), (5, 8), (4, 64), (9, 100), (6, 511), (3, 512), (7, 513), (2, 1024), (5, 1030), (3, 2048), (300, 2056),
          (3, 4096), (261, 4099), (3, 4999), (2, 8192), (258, 8192), (2, 8200), (3, 16384), (2, 16390), (2, 33000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad", [0, 5])
def test_forward(rows, cols, dtype, pad):
    gen = R.generator(rows, cols, dtype, pad)
    x, w = R.rows(gen, rows, cols, dtype, pad), R.rows(gen, 1, cols, dtype)[0]
    r = R.rows(gen, rows, cols, dtype, pad, 3.0) if (rows + cols) % 2 or pad else None
    f = layer().tg_rms_norm(x, w, residual=r, eps=EPS)
    h, rstd, y = norm(x, w, r)
    size = h.abs() if r is None else R.f64(x).abs() + R.f64(r).abs()
    grow = stat_error(cols) + 8 * E32
    # h may cancel: its own error is e of the larger addend
    slack = 2 * E32 * size
    R.within(f.y, y, 1.01 * U[dtype] * y.abs() + grow * y.abs() + slack * rstd * R.f64(w).abs() + TINY[dtype], "y")
    R.within(f.rstd, rstd[:, 0], (grow + 4 * E32) * rstd[:, 0], "rstd")
    if r is None:
        assert f.hidden is x
    else:
        R.within(f.hidden, h, 1.01 * U[dtype] * h.abs() + slack + TINY[dtype], "hidden")


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_forward_in_8_bits(rows, cols, dtype):
    gen = R.generator("e4m3", rows, cols, dtype)
    x, w, r = R.rows(gen, rows, cols, dtype, 3), R.rows(gen, 1, cols, dtype)[0], R.rows(gen, rows, cols, dtype)
    f = layer().tg_rms_norm(x, w, residual=r, eps=EPS, out_dtype=E4M3)
    h, rstd, y = norm(x, w, r)
    most = y.abs().amax(1)
    slack = 2 * E32 * (R.f64(x).abs() + R.f64(r).abs()) * rstd * R.f64(w).abs()
    R.within(f.scale, most / 448, (stat_error(cols) + 12 * E32) * most / 448 + slack.amax(1) / 448, "scale")
    # half a step: 2^-4 of the value, 2^-10 of the scale below 2^-6
    got = R.f64(f.y.float()) * R.f64(f.scale)[:, None]
    R.within(got, y, (2.0 ** -4 * 1.001) * y.abs() + 2.0 ** -10 * 1.001 * R.f64(f.scale)[:, None] + 2 * slack, "y")
    assert float(f.y.float().abs().max()) <= 448.0


@pytest.mark.parametrize("rows,cols", SHAPES + [(0, 40), (700, 72), (1030, 513), (1100, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad", [0, 5])
def test_gradients(rows, cols, dtype, pad):
    gen = R.generator("grad", rows, cols, dtype, pad)
    hid, w = R.rows(gen, rows, cols, dtype, pad), (1 + R.rows(gen, 1, cols, F32)[0] * 0.2).to(dtype)
    dy = R.rows(gen, rows, cols, dtype, pad)
    dh = R.rows(gen, rows, cols, dtype, pad) if (rows + cols) % 2 else None
    h = R.f64(hid)
    rstd = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    given = rstd[:, 0].float().cuda()
    dx, dw = layer().tg_rms_norm_grad(dy, hid, w, given, dhidden=dh)
    s = R.f64(given)[:, None]
    g, xhat = R.f64(dy) * R.f64(w), h * s
    mean, size = (g * xhat).mean(1, keepdim=True), (g * xhat).abs().mean(1, keepdim=True)
    want = s * (g - xhat * mean) + (0 if dh is None else R.f64(dh))
    err = s * (xhat.abs() * (stat_error(cols) * size + 8 * E32 * mean.abs()) + 8 * E32 * g.abs()) + 8 * E32 * want.abs()
    R.within(dx, want, 1.01 * U[dtype] * want.abs() + 2 * err + TINY[dtype], "dx")
    term = R.f64(dy) * xhat
    R.within(dw, term.sum(0), 1.01 * U[dtype] * term.sum(0).abs() + (rows + 16) * E32 * term.abs().sum(0) + TINY[dtype], "dweight")


def test_gradient_against_differences():
    gen = R.generator("differences")
    rows, cols, step = 3, 37, 1e-5
    x, w, dy = R.rows(gen, rows, cols, F32), R.rows(gen, 1, cols, F32)[0], R.rows(gen, rows, cols, F32)
    f = layer().tg_rms_norm(x, w, eps=EPS)
    dx, dw = layer().tg_rms_norm_grad(dy, f.hidden, w, f.rstd)
    at = {"x": R.f64(x), "w": R.f64(w)}

    def loss():
        h = at["x"]
        return float((R.f64(dy) * h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * at["w"]).sum())

    for key, got in (("x", dx), ("w", dw)):
        for i in range(0, at[key].numel(), 5):
            flat = at[key].reshape(-1)
            keep = float(flat[i])
            flat[i] = keep + step
            up = loss()
            flat[i] = keep - step
            down = loss()
            flat[i] = keep
            # the third derivative is of order 1, rounding of the loss about 1e-15 / step
            assert abs((up - down) / (2 * step) - float(got.reshape(-1)[i])) <= 2e-5, (key, i)


def test_zero_rows_and_rows_that_are_not_finite():
    L = layer()
    x = torch.ones(6, 700, device="cuda", dtype=BF16)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 699] = float("inf")
    w = torch.ones(700, device="cuda", dtype=BF16)
    y = L.tg_rms_norm(x, w).y
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[2]).all())
    assert bool((y[3, :699] == 0).all()) and bool(torch.isnan(y[3, 699]))
    assert bool(torch.isfinite(y[[0, 4, 5]]).all())
    f = L.tg_rms_norm(x, w, out_dtype=E4M3)
    q = f.y.float()
    assert float(f.scale[1]) == 1.0 and bool((q[1] == 0).all()) and bool(torch.isnan(q[2]).all())
    assert float(f.scale[3]) == 1.0 and bool(torch.isnan(q[3, 699])) and bool((q[3, :699] == 0).all())
    assert bool((q[[0, 4, 5]] == 448).all())


def test_empty_rows_and_no_columns():
    L = layer()
    w = torch.ones(40, device="cuda")
    f = L.tg_rms_norm(torch.ones(0, 40, device="cuda"), w)
    assert f.y.shape == (0, 40)
    dx, dw = L.tg_rms_norm_grad(f.y, f.hidden, w, f.rstd)
    assert dx.shape == (0, 40) and bool((dw == 0).all())
    f = L.tg_rms_norm(torch.ones(3, 0, device="cuda"), w[:0])
    assert f.y.shape == (3, 0) and f.rstd.shape == (3,)


def test_rows_further_apart_than_32_bits_reach():
    L = layer()
    gen = R.generator("far")
    ld = 1 << 31
    small, w = R.rows(gen, 3, 300, BF16), R.rows(gen, 1, 300, BF16)[0]
    far = torch.empty(2 * ld + 300, dtype=BF16, device="cuda").as_strided((3, 300), (ld, 1))
    far.copy_(small)
    a, b = L.tg_rms_norm(far, w), L.tg_rms_norm(small, w)
    assert torch.equal(a.y, b.y)
    for p, q in zip(L.tg_rms_norm_grad(far, far, w, a.rstd), L.tg_rms_norm_grad(small, small, w, b.rstd)):
        assert torch.equal(p, q)


def test_repeatable_and_replayed():
    L = layer()
    gen = R.generator("graph")
    x, w, r = R.rows(gen, 700, 1000, BF16), R.rows(gen, 1, 1000, BF16)[0], R.rows(gen, 700, 1000, BF16)

    def step():
        f = L.tg_rms_norm(x, w, residual=r)
        return (f.y, f.hidden, f.rstd, *L.tg_rms_norm_grad(x, f.hidden, w, f.rstd, dhidden=r))

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
    bad = [lambda: L.tg_rms_norm(x.double(), w), lambda: L.tg_rms_norm(x, w[:7]), lambda: L.tg_rms_norm(x, w.half()),
           lambda: L.tg_rms_norm(x, w, out_dtype=torch.float16), lambda: L.tg_rms_norm(x, w, residual=x[:2]),
           lambda: L.tg_rms_norm(x.t(), w[:4]), lambda: L.tg_rms_norm(x[0], w), lambda: L.tg_rms_norm(x.cpu(), w),
           lambda: L.tg_rms_norm_grad(x, x, w, w)]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {k} was taken")
    from paper_2606_16907_amd.tangram import TangramError
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(TangramError, match="eps"):
            L.tg_rms_norm(x, w, eps=eps)
