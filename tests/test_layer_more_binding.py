"""The C ABI of the gated projections, the block-scaled product, its quantiser and the layer norm on the CPU: struct
layouts, packed arguments, and the refusals that come before any device call."""
import ctypes
import os
import subprocess

import pytest

from tests.test_layer_binding import ROOT, layer, refused

STRUCTS = ("tg_gated_args", "tg_gated_grad_args", "tg_block_linear_args", "tg_quantize_args", "tg_layer_norm_args",
           "tg_layer_norm_grad_args")


def of(L, name):
    return getattr(L, "".join(w.capitalize() for w in name.split("_")))


def test_structs_match_the_c_compiler(tmp_path):
    L = layer()
    src, lines, want = tmp_path / "layout.c", [], []
    for name in STRUCTS:
        t = of(L, name)
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in t._fields_]
        want += [ctypes.sizeof(t)] + [getattr(t, f).offset for f, _ in t._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tangram_layer.h"\nint main(void){' + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == want


@pytest.mark.parametrize("name", STRUCTS)
def test_packed_arguments_are_the_structure(name):
    L = layer()
    t, pack = of(L, name), getattr(L, "_pack_" + name[3:-5])
    values = [1.5 if kind is ctypes.c_float else 7 * i + 1 for i, (_, kind) in enumerate(t._fields_)]
    packed = pack(*values)
    assert packed == bytes(t(*values))[:len(packed)] and len(packed) > ctypes.sizeof(t) - 8


def gated_args(L, **kw):
    base = dict(x=4096, w_gate=8192, w_up=12288, y=65536, m=4, n=6, k=8, ldx=8, ldwg=8, ldwu=8, ldy=6, ldg=6, ldu=6, type=1, out_type=1)
    return L.TgGatedArgs(**{**base, **kw})


@pytest.mark.parametrize("change,word", [
    (dict(type=0, out_type=0), "type"), (dict(out_type=2), "type"), (dict(type=3, out_type=0), "type"), (dict(type=4), "type"), (dict(act=4), "act"),
    (dict(m=-1), "m -1"), (dict(n=1 << 20), "n 1048576"), (dict(k=1 << 21), "k 2097152"), (dict(reserved=1), "reserved"), (dict(x=None), "x is NULL"),
    (dict(w_up=None), "w_up is NULL"), (dict(w_gate=8193), "aligned"), (dict(ldwu=7), "stride"), (dict(ldy=5), "stride"), (dict(y=None), "y is NULL"),
    (dict(gate=65536), "together"), (dict(gate=65536, up=131072, ldu=3), "stride"), (dict(up_bias=3), "aligned"), (dict(x_scale=4096), "together"),
    (dict(x_scale=4096, gate_scale=4096, up_scale=4096), "8-bit"), (dict(type=3, x_scale=4096, gate_scale=4096, up_scale=4098), "aligned")])
def test_gated_refuses(change, word):
    L = layer()
    refused(L.load_library().tg_gated(gated_args(L, **change), None, 0, None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(type=0), "type"), (dict(act=-1), "act"), (dict(k=-2), "k -2"), (dict(dy=None), "dy is NULL"), (dict(gate=None), "gate is NULL"),
    (dict(up=4097), "aligned"), (dict(w_gate=None), "w_gate is NULL"), (dict(x=None), "x is NULL"), (dict(dw_up=4097), "aligned"), (dict(lddx=3), "stride"),
    (dict(dgate_bias=5), "aligned"), (dict(ldg=2), "stride")])
def test_gated_grad_refuses(change, word):
    L = layer()
    base = dict(dy=4096, gate=4096, up=4096, x=8192, w_gate=12288, w_up=12288, dx=65536, dw_gate=131072, dw_up=196608, m=4, n=6, k=8, lddy=6, ldg=6, ldu=6,
                ldx=8, ldwg=8, ldwu=8, lddx=8, lddwg=8, lddwu=8, type=1)
    refused(L.load_library().tg_gated_grad(L.TgGatedGradArgs(**{**base, **change}), None, 0, None), word)


@pytest.mark.parametrize("change,word", [
    (dict(scale_type=1), "scale_type"), (dict(out_type=0), "out_type"), (dict(out_type=3), "out_type"), (dict(act=9), "act"), (dict(m=-1), "m -1"),
    (dict(reserved=2), "reserved"), (dict(x=None), "x is NULL"), (dict(ldw=100), "stride"), (dict(x_scale=None), "x_scale is NULL"),
    (dict(w_scale=4098), "aligned"), (dict(ldxs=2), "row stride"), (dict(ldxs=1 << 21), "row stride"), (dict(n=300, ldy=300, ldws=2), "row stride"),
    (dict(y=None), "y is NULL"), (dict(residual=65537), "aligned"), (dict(bias=1), "aligned")])
def test_block_linear_refuses(change, word):
    L = layer()
    base = dict(x=4096, w=8192, x_scale=4096, w_scale=8192, y=65536, m=4, n=6, k=300, ldx=300, ldw=300, ldxs=3, ldws=3, ldr=6, ldy=6, out_type=1)
    refused(L.load_library().tg_block_linear(L.TgBlockLinearArgs(**{**base, **change}), None, 0, None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(scale_type=2), "scale_type"), (dict(block_rows=64), "block_rows"), (dict(rows=-1), "rows"), (dict(cols=1 << 31), "cols"),
    (dict(x=None), "x is NULL"), (dict(y=None), "y is NULL"), (dict(scale=None), "scale is NULL"), (dict(x=4097), "aligned"), (dict(scale=4098), "aligned"),
    (dict(ldx=200), "x: row stride"), (dict(ldy=200), "y: row stride"), (dict(lds=2), "scale: row stride"), (dict(reserved=1), "reserved")])
def test_quantize_refuses(change, word):
    L = layer()
    base = dict(x=4096, y=8192, scale=12288, rows=4, cols=300, ldx=300, ldy=300, lds=3, type=1, scale_type=0, block_rows=1)
    refused(L.load_library().tg_quantize(L.TgQuantizeArgs(**{**base, **change}), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(out_type=0), "out_type"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(rows=-1), "rows"),
    (dict(cols=1 << 31), "cols"), (dict(x=None), "x is NULL"), (dict(weight=None), "weight is NULL"), (dict(bias=4097), "aligned"), (dict(ldx=3), "stride"),
    (dict(out_type=3), "scale is NULL"), (dict(scale=4096), "scale"), (dict(mean=4098), "aligned"), (dict(rstd=4098), "aligned"), (dict(reserved=1), "reserved")])
def test_layer_norm_refuses(change, word):
    L = layer()
    base = dict(x=4096, weight=8192, y=65536, rows=4, cols=8, ldx=8, ldr=8, ldh=8, ldy=8, eps=1e-6, type=1, out_type=1)
    refused(L.load_library().tg_layer_norm(L.TgLayerNormArgs(**{**base, **change}), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(rows=-1), "rows"), (dict(mean=None), "mean is NULL"), (dict(rstd=None), "rstd is NULL"), (dict(dweight=None), "dweight is NULL"),
    (dict(dbias=4097), "aligned"), (dict(dx=None), "dx is NULL"), (dict(lddy=2), "stride"), (dict(dhidden=4097), "aligned"), (dict(reserved=2), "reserved")])
def test_layer_norm_grad_refuses(change, word):
    L = layer()
    base = dict(dy=4096, hidden=8192, weight=8192, mean=4096, rstd=4096, dx=65536, dweight=4096, rows=4, cols=8, lddy=8, lddh=8, ldh=8, lddx=8, type=1)
    refused(L.load_library().tg_layer_norm_grad(L.TgLayerNormGradArgs(**{**base, **change}), None, 0, None), word)


def test_workspaces_are_checked_before_any_launch():
    from paper_2606_16907_amd import tangram as T
    L = layer()
    lib = L.load_library()
    calls = [
        (lib.tg_gated, lib.tg_gated_workspace_bytes, gated_args(L, m=300, n=300, k=301, ldx=301, ldwg=301, ldwu=301, ldy=300)),
        (lib.tg_gated_grad, lib.tg_gated_grad_workspace_bytes,
         L.TgGatedGradArgs(dy=4096, gate=4096, up=4096, x=8192, w_gate=12288, w_up=12288, dx=65536, dw_gate=131072, dw_up=196608, dgate_bias=4096, m=4, n=6,
                           k=8, lddy=6, ldg=6, ldu=6, ldx=8, ldwg=8, ldwu=8, lddx=8, lddwg=8, lddwu=8, type=1, act=2)),
        (lib.tg_block_linear, lib.tg_block_linear_workspace_bytes,
         L.TgBlockLinearArgs(x=4096, w=8192, x_scale=4096, w_scale=8192, y=65536, m=300, n=300, k=301, ldx=301, ldw=301, ldxs=3, ldws=3, ldy=300, out_type=1)),
        (lib.tg_layer_norm_grad, lib.tg_layer_norm_grad_workspace_bytes,
         L.TgLayerNormGradArgs(dy=4096, hidden=8192, weight=8192, mean=4096, rstd=4096, dx=65536, dweight=4096, dbias=4096, rows=400, cols=8, lddy=8, ldh=8,
                               lddx=8, type=1))]
    for call, size, a in calls:
        need = size(a)
        assert need > 0
        assert call(a, 4096, need - 1, None) == T.TG_ENOMEM and "needed" in T.last_error()
        assert call(a, None, need, None) == T.TG_ENOMEM
        refused(call(a, 4100, need, None), "256-byte")
        assert size(None) == 0


def test_sizes_that_do_not_fit_want_no_workspace():
    L = layer()
    lib = L.load_library()
    assert lib.tg_gated_workspace_bytes(gated_args(L, n=1 << 21)) == 0 and lib.tg_gated_workspace_bytes(gated_args(L, m=-1)) == 0
    assert lib.tg_block_linear_workspace_bytes(L.TgBlockLinearArgs(m=1, n=1, k=1 << 22)) == 0
    assert lib.tg_layer_norm_grad_workspace_bytes(L.TgLayerNormGradArgs(rows=-1, cols=4)) == 0
