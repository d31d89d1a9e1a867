"""The layer operators' C ABI on the CPU: exports, struct layouts, and the
refusals that come before any device call."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "tangram_layer.h")
STRUCTS = ("tg_linear_args", "tg_linear_grad_args", "tg_rms_norm_args", "tg_rms_norm_grad_args", "tg_adamw_tensor",
           "tg_adamw_rates")


def layer():
    from paper_2606_16907_amd import layer as L
    L.load_library()
    return L


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(tg_[a-z_]+)\s*\(", text)))


def test_binding_declares_every_export():
    L = layer()
    assert sorted(L.EXPORTS) == declared()
    lib = L.load_library()
    assert all(hasattr(lib, n) for n in declared())


def test_structs_match_the_c_compiler(tmp_path):
    L = layer()
    src = tmp_path / "layout.c"
    types = [getattr(L, "".join(w.capitalize() for w in s.split("_"))) for s in STRUCTS]
    lines = []
    for name, t in zip(STRUCTS, types):
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in t._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tangram_layer.h"\nint main(void){' + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    want = []
    for t in types:
        want.append(ctypes.sizeof(t))
        want += [getattr(t, f).offset for f, _ in t._fields_]
    assert got == want


def refused(status, word):
    from paper_2606_16907_amd import tangram as T
    assert status == T.TG_EINVAL
    assert word in T.last_error(), T.last_error()


def linear_args(L, **kw):
    base = dict(x=4096, w=8192, y=65536, m=4, n=6, k=8, ldx=8, ldw=8, ldr=6, ldy=6, ldp=6, type=1, out_type=1)
    return L.TgLinearArgs(**{**base, **kw})


@pytest.mark.parametrize("change,word", [
    (dict(type=0, out_type=0), "type"), (dict(out_type=2), "type"), (dict(type=3, out_type=0), "type"), (dict(type=9), "type"),
    (dict(act=4), "act"), (dict(act=-1), "act"), (dict(m=-1), "m -1"), (dict(n=1 << 31), "n 2147483648"), (dict(reserved=1), "reserved"),
    (dict(x=None), "x is NULL"), (dict(x=4097), "aligned"), (dict(ldx=7), "stride"), (dict(ldw=-8), "stride"), (dict(ldy=5), "stride"),
    (dict(y=None), "y is NULL"), (dict(pre=65537), "aligned"), (dict(residual=65536, ldr=2), "stride"), (dict(bias=3), "aligned"),
    (dict(x_scale=4096), "together"), (dict(x_scale=4096, w_scale=4096), "8-bit"),
    (dict(type=3, x_scale=4098, w_scale=4096), "aligned")])
def test_linear_refuses(change, word):
    L = layer()
    refused(L.load_library().tg_linear(linear_args(L, **change), None, 0, None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(type=0), "type"), (dict(act=7), "act"), (dict(k=-2), "k -2"), (dict(dy=None), "dy is NULL"),
    (dict(act=3), "pre is NULL"), (dict(w=None), "w is NULL"), (dict(dw=4097), "aligned"), (dict(lddx=3), "stride"),
    (dict(dbias=5), "aligned")])
def test_linear_grad_refuses(change, word):
    L = layer()
    base = dict(dy=4096, x=8192, w=12288, dx=65536, dw=131072, m=4, n=6, k=8, lddy=6, ldp=6, ldx=8, ldw=8, lddx=8, lddw=8, type=1)
    refused(L.load_library().tg_linear_grad(L.TgLinearGradArgs(**{**base, **change}), None, 0, None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(out_type=0), "out_type"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(rows=-1), "rows"), (dict(cols=1 << 31), "cols"), (dict(x=None), "x is NULL"), (dict(weight=None), "weight is NULL"),
    (dict(ldx=3), "stride"), (dict(y=4097), "aligned"), (dict(out_type=3), "scale is NULL"), (dict(scale=4096), "scale"),
    (dict(rstd=4098), "aligned"), (dict(reserved=1), "reserved"), (dict(hidden=4096, ldh=7), "stride")])
def test_rms_norm_refuses(change, word):
    L = layer()
    base = dict(x=4096, weight=8192, y=65536, rows=4, cols=8, ldx=8, ldr=8, ldh=8, ldy=8, eps=1e-6, type=1, out_type=1)
    refused(L.load_library().tg_rms_norm(L.TgRmsNormArgs(**{**base, **change}), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(rows=-1), "rows"), (dict(rstd=None), "rstd is NULL"), (dict(dweight=None), "dweight is NULL"),
    (dict(dx=None), "dx is NULL"), (dict(lddy=2), "stride"), (dict(dhidden=4097), "aligned"), (dict(reserved=2), "reserved")])
def test_rms_norm_grad_refuses(change, word):
    L = layer()
    base = dict(dy=4096, hidden=8192, weight=8192, rstd=4096, dx=65536, dweight=4096, rows=4, cols=8, lddy=8, lddh=8, ldh=8, lddx=8, type=1)
    refused(L.load_library().tg_rms_norm_grad(L.TgRmsNormGradArgs(**{**base, **change}), None, 0, None), word)


def test_workspaces_are_checked_before_any_launch():
    from paper_2606_16907_amd import tangram as T
    L = layer()
    lib = L.load_library()
    a = L.TgRmsNormGradArgs(dy=4096, hidden=8192, weight=8192, rstd=4096, dx=65536, dweight=4096, rows=4, cols=8, lddy=8, ldh=8, lddx=8,
                            type=1)
    need = lib.tg_rms_norm_grad_workspace_bytes(a)
    assert need >= 4 * 8 * 4
    assert lib.tg_rms_norm_grad(a, 4096, need - 1, None) == T.TG_ENOMEM and "needed" in T.last_error()
    refused(lib.tg_rms_norm_grad(a, 4100, need, None), "256-byte")
    g = L.TgLinearGradArgs(dy=4096, pre=4096, x=8192, w=12288, dx=65536, dw=131072, dbias=4096, m=4, n=6, k=8, lddy=6, ldp=6, ldx=8, ldw=8,
                           lddx=8, lddw=8, type=1, act=3)
    need = lib.tg_linear_grad_workspace_bytes(g)
    assert need >= 4 * 6 * 2 + 6 * 4
    assert lib.tg_linear_grad(g, 4096, need - 1, None) == T.TG_ENOMEM
    assert lib.tg_linear_grad(g, None, need, None) == T.TG_ENOMEM


@pytest.mark.parametrize("change,args,word", [
    (dict(n=-1), (1, 0, 0, 32), "n = -1"), (dict(param=None), (1, 0, 0, 32), "NULL"), (dict(m=4098), (1, 0, 0, 32), "aligned"),
    (dict(), (1, 0, 0, 16), "state_bits"), (dict(), (1, 3, 3, 32), "param_type"), (dict(), (1, 1, 2, 32), "grad_type"),
    (dict(), (1, 0, 0, 8), "scale"), (dict(master=4096), (1, 0, 0, 32), "master"), (dict(), (-1, 0, 0, 32), "n_tensors"),
    (dict(n=1 << 40), (1, 0, 0, 32), "too many")])
def test_adamw_create_refuses(change, args, word):
    L = layer()
    base = dict(param=4096, grad=8192, m=12288, v=16384, n=10)
    table = (L.TgAdamwTensor * 1)(L.TgAdamwTensor(**{**base, **change}))
    out = ctypes.c_void_p(5)
    n, p, g, bits = args
    refused(L.load_library().tg_adamw_create(table, n, p, g, bits, ctypes.byref(out)), word)
    assert out.value is None


def test_binding_refuses_host_tensors():
    import torch
    L = layer()
    t = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        L.tg_linear(t, t)
