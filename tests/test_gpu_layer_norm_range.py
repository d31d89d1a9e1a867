"""The norm at the ends of its range: rows of subnormal numbers, very many columns, outputs in the place of inputs."""
import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E4M3, E32, U

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def layer():
    from paper_2606_16907_amd import layer as L
    return L


@pytest.mark.parametrize("cols", [40, 3000, 33000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_8_bits_of_rows_whose_scale_would_be_subnormal(cols, dtype):
    """|y| from 2^-149 to 2^-100: the scale is no less than 2^-126, so no code passes 448, and scale times code is within
    half a step of the code (2^-4 of it, 2^-10 of the scale below 2^-6) of y."""
    gen = R.generator("subnormal", cols, dtype)
    # first, a row whose largest is 668 of the smallest numbers: over a scale of one of them no code holds it
    exponents = (-149, -146, -142, -141, -140, -139, -133, -130, -126, -120, -118, -117, -110, -100)
    small = [382 * 2.0 ** -149] + [2.0 ** e for e in exponents]
    # rows of +-1 have rstd = 1 - 5e-7 and y = +-weight; the weight's largest element sets the row's scale
    for top in small:
        x = torch.where(torch.rand(2, cols, generator=gen) < 0.5, -1.0, 1.0).to(dtype).cuda()
        w = (torch.rand(cols, generator=gen, dtype=torch.float64) * top).to(dtype)
        w[0] = top * 1.75
        w = w.cuda()
        f = layer().tg_rms_norm(x, w, out_dtype=E4M3)
        y = R.f64(x) * R.f64(w) * (1 + 1e-6) ** -0.5
        got, scale = R.f64(f.y.float()), R.f64(f.scale)[:, None]
        assert bool(torch.isfinite(got).all()), top
        # the kernel's own y is a subnormal of 2^-149 where it is one at all
        bound = (2.0 ** -4 * 1.001) * y.abs() + 2.0 ** -10 * 1.001 * scale + 2.0 ** -149 + (cols / 64 + 40) * E32 * y.abs()
        R.within(got * scale, y, bound, f"top {top}")
        assert bool((scale >= 2.0 ** -126).all()), top


def test_the_gradient_of_half_a_billion_columns():
    """A pattern of 1033 columns, over and over: sums over a row are the pattern's, the weight's gradient repeats too."""
    period, times = 1033, 519721
    cols = period * times
    assert cols > 1 << 29
    gen = R.generator("wide")
    dy, h, w = (R.rows(gen, m, period, BF16) for m in (2, 2, 1))
    rstd = torch.tensor([0.75, 1.25], device="cuda")
    dx, dw = layer().tg_rms_norm_grad(dy.repeat(1, times), h.repeat(1, times), w[0].repeat(times), rstd)
    s = R.f64(rstd)[:, None]
    g, xhat = R.f64(dy) * R.f64(w), R.f64(h) * s
    mean, size = (g * xhat).mean(1, keepdim=True), (g * xhat).abs().mean(1, keepdim=True)
    want = s * (g - xhat * mean)
    # 1024 threads add up a row, cols / 1024 products each, one rounding an addition and one a product
    bound = s * (xhat.abs() * ((cols / 1024 + 32) * E32 * size + 8 * E32 * mean.abs()) + 8 * E32 * g.abs())
    bound = bound + (8 * E32 + 1.01 * U[BF16]) * want.abs()
    term = R.f64(dy) * xhat
    dw_bound = 1.01 * U[BF16] * term.sum(0).abs() + 18 * E32 * term.abs().sum(0)
    for got, want, bound in ((dx, want, bound), (dw[None], term.sum(0)[None], dw_bound[None])):
        for row in range(got.shape[0]):
            far = (got[row].view(times, period).float() - want[row].float().cuda()).abs_()
            # the oracle was rounded to 32 bits for this
            assert bool((far <= (bound[row] + 2 * E32 * want[row].abs()).float().cuda()).all()), row


WIDTHS = [1, 999, 1000, 16390, 33000]  # kept in registers, and read again for each pass


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_dx_in_the_place_of_dy_or_dhidden(cols, dtype):
    L = layer()
    gen = R.generator("alias", cols, dtype)
    rows = 700 if cols < 2000 else 3
    dy, hidden, dh = (R.rows(gen, rows, cols, dtype, 3) for _ in range(3))
    w, rstd = R.rows(gen, 1, cols, dtype)[0], 0.5 + torch.rand(rows, generator=gen).cuda()
    dx, dw = L.tg_rms_norm_grad(dy, hidden, w, rstd, dhidden=dh)
    for which in (0, 1):
        buffers = [dy.clone(), dh.clone()]
        got, dweight = L.tg_rms_norm_grad(buffers[0], hidden, w, rstd, dhidden=buffers[1], dx=buffers[which])
        assert got is buffers[which] and torch.equal(got, dx) and torch.equal(dweight, dw)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_hidden_in_the_place_of_x_or_residual(cols, dtype, eight):
    """The C call's form; the binding allocates hidden."""
    from paper_2606_16907_amd import tangram as T
    L = layer()
    gen = R.generator("hidden", cols, dtype)
    rows = 700 if cols < 2000 else 3
    x, r = R.rows(gen, rows, cols, dtype), R.rows(gen, rows, cols, dtype)
    w = R.rows(gen, 1, cols, dtype)[0]
    want = L.tg_rms_norm(x, w, residual=r, out_dtype=E4M3 if eight else dtype, keep_rstd=True)
    for which in (0, 1):
        b = [x.clone(), r.clone()]
        y, rstd = torch.empty_like(want.y), torch.empty_like(want.rstd)
        scale = torch.empty_like(want.scale) if eight else None
        a = L.TgRmsNormArgs(x=b[0].data_ptr(), residual=b[1].data_ptr(), weight=w.data_ptr(), hidden=b[which].data_ptr(), y=y.data_ptr(),
                            scale=scale.data_ptr() if eight else None, rstd=rstd.data_ptr(), rows=rows, cols=cols, ldx=cols, ldr=cols,
                            ldh=cols, ldy=cols, eps=1e-6, type=L.TYPES[dtype], out_type=L.TYPES[y.dtype])
        T._check(L.load_library().tg_rms_norm(a, torch.cuda.current_stream().cuda_stream), "tg_rms_norm")
        assert torch.equal(b[which], want.hidden) and torch.equal(y.view(torch.uint8), want.y.view(torch.uint8))
        assert torch.equal(rstd, want.rstd) and (not eight or torch.equal(scale, want.scale))
        assert torch.equal(b[1 - which], (x, r)[1 - which])


@pytest.mark.parametrize("rows,cols", [((1 << 22) + 5, 8), ((1 << 20) + 3, 1025)])
def test_more_rows_than_a_launch_takes(rows, cols):
    """Rows repeat, so every row of the result is that of the first ones, and the weight's gradient adds up all of them."""
    L, period = layer(), 16
    gen = R.generator("many rows", rows, cols)
    x, r, dy = (R.rows(gen, period, cols, BF16) for _ in range(3))
    w = R.rows(gen, 1, cols, BF16)[0]
    which = torch.arange(rows, device="cuda") % period
    few, many = L.tg_rms_norm(x, w, residual=r), L.tg_rms_norm(x[which], w, residual=r[which])
    for a, b in ((few.y, many.y), (few.hidden, many.hidden), (few.rstd, many.rstd)):
        assert torch.equal(a[which], b)
    eight = L.tg_rms_norm(x, w, residual=r, out_dtype=E4M3), L.tg_rms_norm(x[which], w, residual=r[which], out_dtype=E4M3)
    assert torch.equal(eight[0].y.view(torch.uint8)[which], eight[1].y.view(torch.uint8))
    assert torch.equal(eight[0].scale[which], eight[1].scale)
    dx, _ = L.tg_rms_norm_grad(dy, few.hidden, w, few.rstd)
    got, dw = L.tg_rms_norm_grad(dy[which], many.hidden, w, many.rstd)
    assert torch.equal(dx[which], got)
    times = torch.bincount(which).double().cpu()[:, None]
    term = times * R.f64(dy) * R.f64(few.hidden) * R.f64(few.rstd)[:, None]
    # 512 blocks add up rows / 512 products each, then 64 of their sums in a strand and 8 strands
    bound = 1.01 * U[BF16] * term.sum(0).abs() + (rows / 512 + 96) * E32 * term.abs().sum(0)
    R.within(dw, term.sum(0), bound, "dweight")
