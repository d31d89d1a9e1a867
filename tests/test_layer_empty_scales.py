"""8-bit products of no rows or no columns take the scales that belong to them: an empty tensor's address is NULL.  On the
CPU, since nothing is launched for an empty output."""
import pytest

from paper_2606_16907_amd import tangram as T
from tests.test_layer_binding import layer, refused

GIVEN = 4096


def linear(L, m, n, x_scale, w_scale, type=3):
    a = L.TgLinearArgs(x=GIVEN if m else None, w=GIVEN if n else None, x_scale=x_scale, w_scale=w_scale, m=m, n=n, k=8, ldx=8, ldw=8, ldy=max(n, 1),
                       type=type, out_type=1)
    return L.load_library().tg_linear(a, None, 0, None)


def gated(L, m, n, x_scale, gate_scale, up_scale, type=3):
    w = GIVEN if n else None
    a = L.TgGatedArgs(x=GIVEN if m else None, w_gate=w, w_up=w, x_scale=x_scale, gate_scale=gate_scale, up_scale=up_scale, m=m, n=n, k=8, ldx=8, ldwg=8,
                      ldwu=8, ldy=max(n, 1), type=type, out_type=1)
    return L.load_library().tg_gated(a, None, 0, None)


@pytest.mark.parametrize("m,n", [(0, 6), (4, 0), (0, 0)])
def test_scales_of_empty_operands(m, n):
    L = layer()
    sx, sw = GIVEN if m else None, GIVEN if n else None
    assert linear(L, m, n, sx, sw) == T.TG_OK
    assert gated(L, m, n, sx, sw, sw) == T.TG_OK
    assert linear(L, m, n, None, None) == T.TG_OK and gated(L, m, n, None, None, None) == T.TG_OK


@pytest.mark.parametrize("m,n", [(0, 6), (4, 0)])
def test_scales_that_are_missing(m, n):
    """Of what is not empty they come together all the same, and with 8-bit inputs alone."""
    L = layer()
    sx, sw = GIVEN if m else None, GIVEN if n else None
    if n:
        refused(gated(L, m, n, sx, sw, None), "together")
        refused(gated(L, m, n, sx, None, sw), "together")
    refused(linear(L, m, n, sx, sw, type=1), "8-bit")
    refused(gated(L, m, n, sx, sw, sw, type=1), "8-bit")


def test_scales_of_operands_that_are_not_empty():
    L = layer()
    refused(linear(L, 4, 6, GIVEN, None), "together")
    refused(linear(L, 4, 6, None, GIVEN), "together")
    for scales in ((None, GIVEN, GIVEN), (GIVEN, None, GIVEN), (GIVEN, GIVEN, None), (GIVEN, None, None), (None, None, GIVEN)):
        refused(gated(L, 4, 6, *scales), "together")
