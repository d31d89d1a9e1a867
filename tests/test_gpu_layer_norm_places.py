"""Layer norms whose hidden rows take the place of an input, at rows that end inside a unit of 16 bytes: the forward kernel
reads such an end together with what lies before it, which another thread writes."""
import ctypes

import pytest
import torch

from tests import layer_ref as R
from tests.layer_ref import E4M3

pytestmark = pytest.mark.gpu
KINDS = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


@pytest.mark.parametrize("place", ["x", "residual"])
@pytest.mark.parametrize("dtype", list(KINDS))
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("rows,cols", [(70, 9), (70, 513), (70, 1001), (300, 1601), (300, 2051), (300, 4099), (300, 8203), (300, 12291), (3, 1001), (3, 12291),
                                       (3, 16381), (3, 40001)])
def test_hidden_in_the_place_of_an_input(rows, cols, eight, dtype, place):
    from paper_2606_16907_amd import layer as L
    gen = R.generator("ln places", rows, cols, eight, dtype)
    x, r, w = R.rows(gen, rows, cols, dtype, 3), R.rows(gen, rows, cols, dtype, 5), R.rows(gen, 1, cols, dtype)[0]
    out = E4M3 if eight else dtype
    want = L.tg_layer_norm(x, w, bias=w, residual=r, out_dtype=out)
    y = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda").view(E4M3) if eight else torch.zeros(rows, cols, dtype=dtype, device="cuda")
    scale = torch.empty(rows, device="cuda")
    hidden = x if place == "x" else r
    a = L.TgLayerNormArgs(x.data_ptr(), r.data_ptr(), w.data_ptr(), w.data_ptr(), hidden.data_ptr(), y.data_ptr(), scale.data_ptr() if eight else None, None, None,
                          rows, cols, x.stride(0), r.stride(0), hidden.stride(0), cols, 1e-5, KINDS[dtype], 3 if eight else KINDS[dtype], 0)
    assert L.load_library().tg_layer_norm(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(hidden, want.hidden)
    assert torch.equal(y.view(torch.uint8) if eight else y, want.y.view(torch.uint8) if eight else want.y)
    assert not eight or torch.equal(scale, want.scale)
