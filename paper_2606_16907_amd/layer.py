"""Binding of the layer operators (include/tangram_layer.h): the feed-forward
half of a planned layer on one GPU.

    y, pre = tg_linear(x, w, bias=b, act="gelu", keep_pre=True)
    dx, dw, db = tg_linear_grad(dy, x, w, pre=pre, act="gelu", bias_grad=True)
    f = tg_rms_norm(x, weight, residual=r)              # f.y, f.hidden, f.rstd
    q = tg_rms_norm(x, weight, residual=r, out_dtype=torch.float8_e4m3fn)
    y = tg_linear(q.y, w8, x_scale=q.scale, w_scale=w8_scale)
    y, gate, up = tg_gated(x, w_gate, w_up, act="silu", keep_pre=True)
    g = tg_gated_grad(dy, x, w_gate, w_up, gate, up, act="silu")    # g.dx, g.dw_gate, g.dw_up
    q, w8 = tg_quantize(x), tg_quantize(w, block_rows=128)
    y = tg_block_linear(q.y, w8.y, q.scale, w8.scale, residual=r)
    f = tg_layer_norm(x, weight, bias=b, residual=r)    # f.y, f.hidden, f.mean, f.rstd
    opt = AdamW(params, grads, *adamw_states(params, bits=8), masters=masters)
    opt.step(step, lr=1e-4, seed=step)

Argument marshalling only, as in the submodule `tangram`: the work is done by
the HIP kernels of libtangram_hip.so on torch's current stream, there is no CPU
fallback, and every buffer is checked here for what a plain pointer cannot
carry.  Matrices are two-dimensional tensors with unit stride along a row and
any row stride.  Outputs are allocated unless they are given.  Nothing is
recorded for autograd: a result never requires a gradient, whatever the inputs
do, and gradients are calls of their own.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple, Optional

import torch

from . import tangram as T

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, E4M3: 3}
SCALE_TYPES = {torch.float32: 0, E8M0: 4}
ACTS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}
SCALE_BLOCK = 256  # consecutive elements of an 8-bit optimizer state that share a scale
BLOCK = 128  # columns (and rows of a weight) of 8-bit values that share a scale

_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t


def _struct(name, **fields):
    return type(name, (ctypes.Structure,), {"_fields_": [(f, t) for names, t in fields.values() for f in names.split()]})


TgLinearArgs = _struct("TgLinearArgs", p=("x w x_scale w_scale bias residual y pre", _vp),
                       n=("m n k ldx ldw ldr ldy ldp", _i64), t=("type out_type act reserved", _i32))
TgLinearGradArgs = _struct("TgLinearGradArgs", p=("dy pre x w dx dw dbias", _vp),
                           n=("m n k lddy ldp ldx ldw lddx lddw", _i64), t=("type act", _i32))
TgRmsNormArgs = _struct("TgRmsNormArgs", p=("x residual weight hidden y scale rstd", _vp),
                        n=("rows cols ldx ldr ldh ldy", _i64), e=("eps", ctypes.c_float),
                        t=("type out_type reserved", _i32))
TgRmsNormGradArgs = _struct("TgRmsNormGradArgs", p=("dy dhidden hidden weight rstd dx dweight", _vp),
                            n=("rows cols lddy lddh ldh lddx", _i64), t=("type reserved", _i32))
TgGatedArgs = _struct("TgGatedArgs", p=("x w_gate w_up x_scale gate_scale up_scale gate_bias up_bias y gate up", _vp),
                      n=("m n k ldx ldwg ldwu ldy ldg ldu", _i64), t=("type out_type act reserved", _i32))
TgGatedGradArgs = _struct("TgGatedGradArgs",
                          p=("dy gate up x w_gate w_up dx dw_gate dw_up dgate_bias dup_bias", _vp),
                          n=("m n k lddy ldg ldu ldx ldwg ldwu lddx lddwg lddwu", _i64), t=("type act", _i32))
TgBlockLinearArgs = _struct("TgBlockLinearArgs", p=("x w x_scale w_scale bias residual y", _vp),
                            n=("m n k ldx ldw ldxs ldws ldr ldy", _i64), t=("scale_type out_type act reserved", _i32))
TgQuantizeArgs = _struct("TgQuantizeArgs", p=("x y scale", _vp), n=("rows cols ldx ldy lds", _i64),
                         t=("type scale_type block_rows reserved", _i32))
TgLayerNormArgs = _struct("TgLayerNormArgs", p=("x residual weight bias hidden y scale mean rstd", _vp),
                          n=("rows cols ldx ldr ldh ldy", _i64), e=("eps", ctypes.c_float),
                          t=("type out_type reserved", _i32))
TgLayerNormGradArgs = _struct("TgLayerNormGradArgs", p=("dy dhidden hidden weight mean rstd dx dweight dbias", _vp),
                              n=("rows cols lddy lddh ldh lddx", _i64), t=("type reserved", _i32))
TgAdamwTensor = _struct("TgAdamwTensor", p=("param grad master m v m_scale v_scale", _vp), n=("n", _i64))
TgAdamwRates = _struct("TgAdamwRates", r=("lr beta1 beta2 eps weight_decay grad_scale", ctypes.c_double),
                       n=("step", _i64), t=("seed reserved", ctypes.c_uint32))

_CODES = {_vp: "Q", _i32: "i", _i64: "q", ctypes.c_float: "f"}


def _packer(args):
    """A function of the structure's fields, NULL as 0, to the bytes of the structure: a third of the time that ctypes
    takes to fill one."""
    return struct.Struct("@" + "".join(_CODES[t] for _, t in args._fields_)).pack


_pack_gated, _pack_gated_grad, _pack_block_linear, _pack_quantize, _pack_layer_norm, _pack_layer_norm_grad = (
    _packer(t) for t in (TgGatedArgs, TgGatedGradArgs, TgBlockLinearArgs, TgQuantizeArgs, TgLayerNormArgs,
                         TgLayerNormGradArgs))

EXPORTS = ("tg_linear_workspace_bytes", "tg_linear", "tg_linear_grad_workspace_bytes", "tg_linear_grad",
           "tg_gated_workspace_bytes", "tg_gated", "tg_gated_grad_workspace_bytes", "tg_gated_grad",
           "tg_block_linear_workspace_bytes", "tg_block_linear", "tg_quantize",
           "tg_rms_norm", "tg_rms_norm_grad_workspace_bytes", "tg_rms_norm_grad",
           "tg_layer_norm", "tg_layer_norm_grad_workspace_bytes", "tg_layer_norm_grad",
           "tg_adamw_create", "tg_adamw_step", "tg_adamw_destroy")

_lib = None
_bytes_calls = {}  # entry points that take their arguments as packed bytes


def load_library():
    """The built library with the layer operators' signatures declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = T.load_library()
    P = ctypes.POINTER
    for name, args in (("tg_linear", TgLinearArgs), ("tg_linear_grad", TgLinearGradArgs),
                       ("tg_gated", TgGatedArgs), ("tg_gated_grad", TgGatedGradArgs),
                       ("tg_block_linear", TgBlockLinearArgs),
                       ("tg_rms_norm_grad", TgRmsNormGradArgs), ("tg_layer_norm_grad", TgLayerNormGradArgs)):
        size = getattr(L, name + "_workspace_bytes")
        size.argtypes, size.restype = [P(args)], _sz
        getattr(L, name).argtypes = [P(args), _vp, _sz, _vp]
    L.tg_rms_norm.argtypes = [P(TgRmsNormArgs), _vp]
    L.tg_layer_norm.argtypes = [P(TgLayerNormArgs), _vp]
    L.tg_quantize.argtypes = [P(TgQuantizeArgs), _vp]
    L.tg_adamw_create.argtypes = [P(TgAdamwTensor), _i32, _i32, _i32, _i32, P(_vp)]
    L.tg_adamw_step.argtypes = [_vp, P(TgAdamwRates), _vp]
    L.tg_adamw_destroy.argtypes, L.tg_adamw_destroy.restype = [_vp], None
    for name in ("tg_gated", "tg_gated_grad", "tg_block_linear", "tg_quantize", "tg_layer_norm", "tg_layer_norm_grad"):
        call = _bytes_calls[name] = L[name]  # an object of its own
        call.argtypes = [ctypes.c_char_p] + getattr(L, name).argtypes[1:]
        if hasattr(L, name + "_workspace_bytes"):
            size = _bytes_calls[name + "_workspace_bytes"] = L[name + "_workspace_bytes"]
            size.argtypes, size.restype = [ctypes.c_char_p], _sz
    _lib = L
    return L


def _elsewhere(t, what, device):
    return ValueError(f"{what}: on {t.device}, the current device cuda:{device} expected")


def _matrix(t, dtype, rows, cols, what, device):
    """Pointer and row stride of a [rows, cols] matrix; any None size is the tensor's own."""
    if t.get_device() != device:
        raise _elsewhere(t, what, device)
    if t.dtype != dtype:
        raise ValueError(f"{what}: dtype {t.dtype}, {dtype} expected")
    if t.dim() != 2:
        raise ValueError(f"{what}: {t.dim()} dimensions, a matrix expected")
    m, n = t.shape
    if (rows is not None and m != rows) or (cols is not None and n != cols):
        raise ValueError(f"{what}: shape {(m, n)}, {(rows, cols)} expected")
    ld, unit = t.stride()
    if n > 1 and unit != 1:
        raise ValueError(f"{what}: unit stride along a row expected, stride {unit}")
    if m > 1 and ld < n:
        raise ValueError(f"{what}: rows overlap (row stride {ld}, length {n})")
    return t.data_ptr(), ld


def _vector(t, dtype, n, what, device):
    if t.get_device() != device:
        raise _elsewhere(t, what, device)
    if t.dtype != dtype:
        raise ValueError(f"{what}: dtype {t.dtype}, {dtype} expected")
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, {n} consecutive elements expected")
    return t.data_ptr()


# torch.cuda.current_stream(device).cuda_stream without the Stream object around it
# (0.1 us in place of 1.2; a call of the smallest kernels takes 10 in all)
_stream = torch._C._cuda_getCurrentRawStream


def _workspace(size, given, like, device):
    """Pointer and size of the given workspace or of a new one, and what keeps it
    until the call is queued: the allocator hands it out again on this stream only."""
    if given is not None:
        return (*T._dws(given, "workspace", device), given)
    if not size:
        return None, 0, None
    t = like.new_empty(size, dtype=torch.uint8)
    return t.data_ptr(), size, t


def _call(name, args, given, like, device):
    """Entry point `name` on packed arguments, with the workspace that it wants."""
    ws, size, _kept = _workspace(_bytes_calls[name + "_workspace_bytes"](args), given, like, device)
    T._check(_bytes_calls[name](args, ws, size, _stream(device)), name)


def _act(act):
    if act not in ACTS:
        raise ValueError(f"act: {act!r}, one of none, relu, silu, gelu expected")
    return ACTS[act]


def _out(out, like, m, n, dtype, device, what="out"):
    """The [m, n] output, its pointer and row stride."""
    if out is None:
        out = like.new_empty((m, n), dtype=dtype)
        return out, out.data_ptr(), n
    return out, *_matrix(out, dtype, m, n, what, device)


def _vector_out(out, like, n, device, what):
    if out is None:
        out = like.new_empty(n)
        return out, out.data_ptr()
    return out, _vector(out, like.dtype, n, what, device)


def tg_linear(x, w, bias=None, act="none", residual=None, x_scale=None, w_scale=None, out_dtype=None,
              keep_pre=False, out=None, workspace=None):
    """act(x w^T + bias) + residual for x [m, k] and w [n, k] in bfloat16,
    float16 or float8_e4m3fn (then x_scale [m] and w_scale [n] floats multiply
    the product, both or neither, and the other operands have out_dtype,
    bfloat16 unless given).  Returns y, or with keep_pre (y, pre) where pre
    holds x w^T + bias, None without an activation: what tg_linear_grad wants.
    `out` receives y and may be the residual."""
    lib = load_library()
    device = torch.cuda.current_device()
    dtype = x.dtype
    if dtype not in TYPES or dtype == torch.float32:
        raise ValueError(f"x: dtype {dtype}, bfloat16, float16 or float8_e4m3fn expected")
    if out_dtype is None:
        out_dtype = torch.bfloat16 if dtype == E4M3 else dtype
    if (out_dtype not in (torch.bfloat16, torch.float16)) or (dtype != E4M3 and out_dtype != dtype):
        raise ValueError(f"out_dtype: {out_dtype} for inputs of {dtype}")
    px, ldx = _matrix(x, dtype, None, None, "x", device)
    m, k = x.shape
    pw, ldw = _matrix(w, dtype, None, k, "w", device)
    n = w.shape[0]
    if (x_scale is None) != (w_scale is None) or (x_scale is not None and dtype != E4M3):
        raise ValueError("x_scale and w_scale come together, with 8-bit inputs")
    psx = None if x_scale is None else _vector(x_scale, torch.float32, m, "x_scale", device)
    psw = None if w_scale is None else _vector(w_scale, torch.float32, n, "w_scale", device)
    pb = None if bias is None else _vector(bias, out_dtype, n, "bias", device)
    pr, ldr = (None, 0) if residual is None else _matrix(residual, out_dtype, m, n, "residual", device)
    act = _act(act)
    y, py, ldy = _out(out, x, m, n, out_dtype, device)
    pre, pp, ldp = _out(None, x, m, n, out_dtype, device) if keep_pre and act else (None, None, 0)
    a = TgLinearArgs(px, pw, psx, psw, pb, pr, py, pp, m, n, k, ldx, ldw, ldr, ldy, ldp, TYPES[dtype],
                     TYPES[out_dtype], act, 0)
    ws, size, _kept = _workspace(lib.tg_linear_workspace_bytes(a), workspace, x, device)
    T._check(lib.tg_linear(a, ws, size, _stream(device)), "tg_linear")
    return (y, pre) if keep_pre else y


def tg_linear_grad(dy, x, w, pre=None, act="none", bias_grad=False, x_grad=True, w_grad=True, dx=None, dw=None,
                   dbias=None, workspace=None):
    """(dx, dw, dbias) of tg_linear from dy [m, n], in the inputs' type; those
    not asked for are None, those given are written to.  The residual's gradient
    is dy.  `pre` is tg_linear's, needed where there is an activation."""
    lib = load_library()
    device = torch.cuda.current_device()
    dtype = dy.dtype
    if dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"dy: dtype {dtype}, bfloat16 or float16 expected")
    pdy, lddy = _matrix(dy, dtype, None, None, "dy", device)
    m, n = dy.shape
    px, ldx = _matrix(x, dtype, m, None, "x", device)
    k = x.shape[1]
    pw, ldw = _matrix(w, dtype, n, k, "w", device)
    act = _act(act)
    if act and pre is None:
        raise ValueError("pre: needed for the gradient of an activation (tg_linear with keep_pre)")
    pp, ldp = _matrix(pre, dtype, m, n, "pre", device) if act else (None, 0)
    dx, pdx, lddx = _out(dx, dy, m, k, dtype, device, "dx") if x_grad else (None, None, 0)
    dw, pdw, lddw = _out(dw, dy, n, k, dtype, device, "dw") if w_grad else (None, None, 0)
    db, pdb = _vector_out(dbias, dy, n, device, "dbias") if bias_grad else (None, None)
    a = TgLinearGradArgs(pdy, pp, px, pw, pdx, pdw, pdb, m, n, k, lddy, ldp, ldx, ldw, lddx, lddw, TYPES[dtype], act)
    ws, size, _kept = _workspace(lib.tg_linear_grad_workspace_bytes(a), workspace, dy, device)
    T._check(lib.tg_linear_grad(a, ws, size, _stream(device)), "tg_linear_grad")
    return dx, dw, db


def tg_gated(x, w_gate, w_up, gate_bias=None, up_bias=None, act="silu", x_scale=None, gate_scale=None, up_scale=None,
             out_dtype=None, keep_pre=False, out=None, workspace=None):
    """act(gate) up with gate = x w_gate^T + gate_bias and up = x w_up^T + up_bias
    for x [m, k] and w_gate, w_up [n, k] in bfloat16, float16 or float8_e4m3fn
    (then x_scale [m], gate_scale [n] and up_scale [n] floats multiply the
    products, all or none, and the other operands have out_dtype, bfloat16 unless
    given).  Returns y, or with keep_pre (y, gate, up): what tg_gated_grad wants."""
    load_library()
    device = torch.cuda.current_device()
    dtype = x.dtype
    if dtype not in TYPES or dtype == torch.float32:
        raise ValueError(f"x: dtype {dtype}, bfloat16, float16 or float8_e4m3fn expected")
    if out_dtype is None:
        out_dtype = torch.bfloat16 if dtype == E4M3 else dtype
    if (out_dtype not in (torch.bfloat16, torch.float16)) or (dtype != E4M3 and out_dtype != dtype):
        raise ValueError(f"out_dtype: {out_dtype} for inputs of {dtype}")
    px, ldx = _matrix(x, dtype, None, None, "x", device)
    m, k = x.shape
    pg, ldwg = _matrix(w_gate, dtype, None, k, "w_gate", device)
    n = w_gate.shape[0]
    pu, ldwu = _matrix(w_up, dtype, n, k, "w_up", device)
    scales = (x_scale, gate_scale, up_scale)
    if any(s is not None for s in scales) and (dtype != E4M3 or any(s is None for s in scales)):
        raise ValueError("x_scale, gate_scale and up_scale come together, with 8-bit inputs")
    psx = 0 if x_scale is None else _vector(x_scale, torch.float32, m, "x_scale", device)
    psg = 0 if gate_scale is None else _vector(gate_scale, torch.float32, n, "gate_scale", device)
    psu = 0 if up_scale is None else _vector(up_scale, torch.float32, n, "up_scale", device)
    pbg = 0 if gate_bias is None else _vector(gate_bias, out_dtype, n, "gate_bias", device)
    pbu = 0 if up_bias is None else _vector(up_bias, out_dtype, n, "up_bias", device)
    act = _act(act)
    y, py, ldy = _out(out, x, m, n, out_dtype, device)
    gate, pgate, ldg = _out(None, x, m, n, out_dtype, device) if keep_pre else (None, 0, 0)
    up, pup, ldu = _out(None, x, m, n, out_dtype, device) if keep_pre else (None, 0, 0)
    a = _pack_gated(px, pg, pu, psx, psg, psu, pbg, pbu, py, pgate, pup, m, n, k, ldx, ldwg, ldwu, ldy, ldg, ldu,
                    TYPES[dtype], TYPES[out_dtype], act, 0)
    _call("tg_gated", a, workspace, x, device)
    return (y, gate, up) if keep_pre else y


class GatedGrads(NamedTuple):
    dx: Optional[torch.Tensor]
    dw_gate: Optional[torch.Tensor]
    dw_up: Optional[torch.Tensor]
    dgate_bias: Optional[torch.Tensor]
    dup_bias: Optional[torch.Tensor]


def tg_gated_grad(dy, x, w_gate, w_up, gate, up, act="silu", bias_grad=False, x_grad=True, w_grad=True, dx=None,
                  dw_gate=None, dw_up=None, dgate_bias=None, dup_bias=None, workspace=None):
    """Gradients of tg_gated from dy [m, n], in the inputs' type; those not asked
    for are None, those given are written to.  `gate` and `up` are tg_gated's."""
    load_library()
    device = torch.cuda.current_device()
    dtype = dy.dtype
    if dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"dy: dtype {dtype}, bfloat16 or float16 expected")
    pdy, lddy = _matrix(dy, dtype, None, None, "dy", device)
    m, n = dy.shape
    px, ldx = _matrix(x, dtype, m, None, "x", device)
    k = x.shape[1]
    pwg, ldwg = _matrix(w_gate, dtype, n, k, "w_gate", device)
    pwu, ldwu = _matrix(w_up, dtype, n, k, "w_up", device)
    pg, ldg = _matrix(gate, dtype, m, n, "gate", device)
    pu, ldu = _matrix(up, dtype, m, n, "up", device)
    act = _act(act)
    dx, pdx, lddx = _out(dx, dy, m, k, dtype, device, "dx") if x_grad else (None, 0, 0)
    dwg, pdwg, lddwg = _out(dw_gate, dy, n, k, dtype, device, "dw_gate") if w_grad else (None, 0, 0)
    dwu, pdwu, lddwu = _out(dw_up, dy, n, k, dtype, device, "dw_up") if w_grad else (None, 0, 0)
    dbg, pdbg = _vector_out(dgate_bias, dy, n, device, "dgate_bias") if bias_grad else (None, 0)
    dbu, pdbu = _vector_out(dup_bias, dy, n, device, "dup_bias") if bias_grad else (None, 0)
    a = _pack_gated_grad(pdy, pg, pu, px, pwg, pwu, pdx, pdwg, pdwu, pdbg, pdbu, m, n, k, lddy, ldg, ldu, ldx, ldwg, ldwu,
                         lddx, lddwg, lddwu, TYPES[dtype], act)
    _call("tg_gated_grad", a, workspace, dy, device)
    return GatedGrads(dx, dwg, dwu, dbg, dbu)


class Quantized(NamedTuple):
    y: torch.Tensor      # float8_e4m3fn
    scale: torch.Tensor  # [ceil(rows / block_rows), ceil(cols / 128)]


def tg_quantize(x, block_rows=1, scale_dtype=torch.float32, out=None, scale=None):
    """8-bit values of float32, bfloat16 or float16 rows with a scale for every 128
    consecutive columns of a row (block_rows 1) or of 128 rows (block_rows 128):
    max |x| / 448 over the block, or with scale_dtype float8_e8m0fnu the least
    power of two that is no smaller.  `out` and `scale` are written to where given."""
    load_library()
    device = torch.cuda.current_device()
    dtype = x.dtype
    if dtype not in TYPES or dtype == E4M3:
        raise ValueError(f"x: dtype {dtype}, float32, bfloat16 or float16 expected")
    if scale_dtype not in SCALE_TYPES:
        raise ValueError(f"scale_dtype: {scale_dtype}, float32 or float8_e8m0fnu expected")
    if block_rows not in (1, BLOCK):
        raise ValueError(f"block_rows: {block_rows}, 1 or {BLOCK} expected")
    px, ldx = _matrix(x, dtype, None, None, "x", device)
    rows, cols = x.shape
    y, py, ldy = _out(out, x, rows, cols, E4M3, device)
    scale, ps, lds = _out(scale, x, -(-rows // block_rows), -(-cols // BLOCK), scale_dtype, device, "scale")
    a = _pack_quantize(px, py, ps, rows, cols, ldx, ldy, lds, TYPES[dtype], SCALE_TYPES[scale_dtype], block_rows, 0)
    T._check(_bytes_calls["tg_quantize"](a, _stream(device)), "tg_quantize")
    return Quantized(y, scale)


def tg_block_linear(x, w, x_scale, w_scale, bias=None, act="none", residual=None, out_dtype=torch.bfloat16, out=None,
                    workspace=None):
    """act(x w^T + bias) + residual for float8_e4m3fn x [m, k] and w [n, k], x with a
    scale for every 128 columns of a row, x_scale [m, ceil(k / 128)], and w for
    every block of 128 x 128, w_scale [ceil(n / 128), ceil(k / 128)], both float32
    or both float8_e8m0fnu.  The other operands have out_dtype, bfloat16 or
    float16.  `out` receives y and may be the residual."""
    load_library()
    device = torch.cuda.current_device()
    if x_scale.dtype not in SCALE_TYPES:
        raise ValueError(f"x_scale: dtype {x_scale.dtype}, float32 or float8_e8m0fnu expected")
    if out_dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"out_dtype: {out_dtype}, bfloat16 or float16 expected")
    px, ldx = _matrix(x, E4M3, None, None, "x", device)
    m, k = x.shape
    pw, ldw = _matrix(w, E4M3, None, k, "w", device)
    n, blocks = w.shape[0], -(-k // BLOCK)
    pxs, ldxs = _matrix(x_scale, x_scale.dtype, m, blocks, "x_scale", device)
    pws, ldws = _matrix(w_scale, x_scale.dtype, -(-n // BLOCK), blocks, "w_scale", device)
    pb = 0 if bias is None else _vector(bias, out_dtype, n, "bias", device)
    pr, ldr = (0, 0) if residual is None else _matrix(residual, out_dtype, m, n, "residual", device)
    y, py, ldy = _out(out, x, m, n, out_dtype, device)
    a = _pack_block_linear(px, pw, pxs, pws, pb, pr, py, m, n, k, ldx, ldw, ldxs, ldws, ldr, ldy,
                           SCALE_TYPES[x_scale.dtype], TYPES[out_dtype], _act(act), 0)
    _call("tg_block_linear", a, workspace, x, device)
    return y


class Norm(NamedTuple):
    y: torch.Tensor
    scale: Optional[torch.Tensor]  # [rows], 8-bit outputs only
    hidden: torch.Tensor           # x + residual; x itself where there is no residual
    rstd: Optional[torch.Tensor]   # [rows], for the gradient


def tg_rms_norm(x, weight, residual=None, eps=1e-6, out_dtype=None, out=None, keep_rstd=None):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight over rows of
    float32, bfloat16 or float16; with out_dtype float8_e4m3fn y is y / scale
    for a scale per row.  rstd, which the gradient takes, is returned with
    outputs in the inputs' type, or as keep_rstd says."""
    lib = load_library()
    device = torch.cuda.current_device()
    dtype = x.dtype
    if dtype not in TYPES or dtype == E4M3:
        raise ValueError(f"x: dtype {dtype}, float32, bfloat16 or float16 expected")
    if out_dtype is None:
        out_dtype = dtype
    if out_dtype not in (dtype, E4M3):
        raise ValueError(f"out_dtype: {out_dtype} for an input of {dtype}")
    px, ldx = _matrix(x, dtype, None, None, "x", device)
    rows, cols = x.shape
    pw = _vector(weight, dtype, cols, "weight", device)
    pr, ldr = (None, 0) if residual is None else _matrix(residual, dtype, rows, cols, "residual", device)
    eight = out_dtype == E4M3
    hidden, ph, ldh = (x, None, 0) if residual is None else _out(None, x, rows, cols, dtype, device)
    y, py, ldy = _out(out, x, rows, cols, out_dtype, device)
    scale = x.new_empty(rows, dtype=torch.float32) if eight else None
    rstd = x.new_empty(rows, dtype=torch.float32) if keep_rstd or (keep_rstd is None and not eight) else None
    a = TgRmsNormArgs(px, pr, pw, ph, py, None if scale is None else scale.data_ptr(),
                      None if rstd is None else rstd.data_ptr(), rows, cols, ldx, ldr, ldh, ldy, eps, TYPES[dtype],
                      TYPES[out_dtype], 0)
    T._check(lib.tg_rms_norm(a, _stream(device)), "tg_rms_norm")
    return Norm(y, scale, hidden, rstd)


def tg_rms_norm_grad(dy, hidden, weight, rstd, dhidden=None, dx=None, dweight=None, workspace=None):
    """(dx, dweight) of tg_rms_norm; dx is the gradient of x and of the residual
    alike.  dhidden is the gradient that arrives at `hidden` from further on; dx
    and dweight are written to where they are given (dx may be dy or dhidden)."""
    lib = load_library()
    device = torch.cuda.current_device()
    dtype = dy.dtype
    if dtype not in TYPES or dtype == E4M3:
        raise ValueError(f"dy: dtype {dtype}, float32, bfloat16 or float16 expected")
    pdy, lddy = _matrix(dy, dtype, None, None, "dy", device)
    rows, cols = dy.shape
    ph, ldh = _matrix(hidden, dtype, rows, cols, "hidden", device)
    pw = _vector(weight, dtype, cols, "weight", device)
    ps = _vector(rstd, torch.float32, rows, "rstd", device)
    pdh, lddh = (None, 0) if dhidden is None else _matrix(dhidden, dtype, rows, cols, "dhidden", device)
    dx, pdx, lddx = _out(dx, dy, rows, cols, dtype, device, "dx")
    dweight, pdw = _vector_out(dweight, dy, cols, device, "dweight")
    a = TgRmsNormGradArgs(pdy, pdh, ph, pw, ps, pdx, pdw, rows, cols, lddy, lddh, ldh, lddx,
                          TYPES[dtype], 0)
    ws, size, _kept = _workspace(lib.tg_rms_norm_grad_workspace_bytes(a), workspace, dy, device)
    T._check(lib.tg_rms_norm_grad(a, ws, size, _stream(device)), "tg_rms_norm_grad")
    return dx, dweight


class LayerNorm(NamedTuple):
    y: torch.Tensor
    scale: Optional[torch.Tensor]  # [rows], 8-bit outputs only
    hidden: torch.Tensor           # x + residual; x itself where there is no residual
    mean: Optional[torch.Tensor]   # [rows], for the gradient
    rstd: Optional[torch.Tensor]   # the same


def tg_layer_norm(x, weight, bias=None, residual=None, eps=1e-5, out_dtype=None, out=None, keep_stats=None):
    """h = x + residual, y = (h - mean(h)) / sqrt(mean((h - mean(h))^2) + eps) *
    weight + bias over rows of float32, bfloat16 or float16; with out_dtype
    float8_e4m3fn y is y / scale for a scale per row.  mean and rstd, which the
    gradient takes, are returned with outputs in the inputs' type, or as keep_stats
    says."""
    load_library()
    device = torch.cuda.current_device()
    dtype = x.dtype
    if dtype not in TYPES or dtype == E4M3:
        raise ValueError(f"x: dtype {dtype}, float32, bfloat16 or float16 expected")
    if out_dtype is None:
        out_dtype = dtype
    if out_dtype not in (dtype, E4M3):
        raise ValueError(f"out_dtype: {out_dtype} for an input of {dtype}")
    px, ldx = _matrix(x, dtype, None, None, "x", device)
    rows, cols = x.shape
    pw = _vector(weight, dtype, cols, "weight", device)
    pb = 0 if bias is None else _vector(bias, dtype, cols, "bias", device)
    pr, ldr = (0, 0) if residual is None else _matrix(residual, dtype, rows, cols, "residual", device)
    eight = out_dtype == E4M3
    hidden, ph, ldh = (x, 0, 0) if residual is None else _out(None, x, rows, cols, dtype, device)
    y, py, ldy = _out(out, x, rows, cols, out_dtype, device)
    scale = mean = rstd = None
    ps = pm = pd = 0
    if eight:
        scale = x.new_empty(rows, dtype=torch.float32)
        ps = scale.data_ptr()
    if keep_stats or (keep_stats is None and not eight):
        mean, rstd = x.new_empty(rows, dtype=torch.float32), x.new_empty(rows, dtype=torch.float32)
        pm, pd = mean.data_ptr(), rstd.data_ptr()
    a = _pack_layer_norm(px, pr, pw, pb, ph, py, ps, pm, pd, rows, cols, ldx, ldr, ldh, ldy, eps, TYPES[dtype],
                         TYPES[out_dtype], 0)
    T._check(_bytes_calls["tg_layer_norm"](a, _stream(device)), "tg_layer_norm")
    return LayerNorm(y, scale, hidden, mean, rstd)


def tg_layer_norm_grad(dy, hidden, weight, mean, rstd, dhidden=None, bias_grad=True, dx=None, dweight=None, dbias=None,
                       workspace=None):
    """(dx, dweight, dbias) of tg_layer_norm, dbias None where it is not asked for;
    dx is the gradient of x and of the residual alike.  dhidden is the gradient that
    arrives at `hidden` from further on; outputs are written to where they are given
    (dx may be dy or dhidden)."""
    load_library()
    device = torch.cuda.current_device()
    dtype = dy.dtype
    if dtype not in TYPES or dtype == E4M3:
        raise ValueError(f"dy: dtype {dtype}, float32, bfloat16 or float16 expected")
    pdy, lddy = _matrix(dy, dtype, None, None, "dy", device)
    rows, cols = dy.shape
    ph, ldh = _matrix(hidden, dtype, rows, cols, "hidden", device)
    pw = _vector(weight, dtype, cols, "weight", device)
    pm, ps = _vector(mean, torch.float32, rows, "mean", device), _vector(rstd, torch.float32, rows, "rstd", device)
    pdh, lddh = (0, 0) if dhidden is None else _matrix(dhidden, dtype, rows, cols, "dhidden", device)
    dx, pdx, lddx = _out(dx, dy, rows, cols, dtype, device, "dx")
    dweight, pdw = _vector_out(dweight, dy, cols, device, "dweight")
    dbias, pdb = _vector_out(dbias, dy, cols, device, "dbias") if bias_grad else (None, 0)
    a = _pack_layer_norm_grad(pdy, pdh, ph, pw, pm, ps, pdx, pdw, pdb, rows, cols, lddy, lddh, ldh, lddx, TYPES[dtype], 0)
    _call("tg_layer_norm_grad", a, workspace, dy, device)
    return dx, dweight, dbias


# ----------------------------------------------------------------------------
# AdamW
# ----------------------------------------------------------------------------
def adamw_states(params, bits=32):
    """Zero moments for `params`: lists (m, v), or with bits=8 (m, v, m_scales, v_scales)."""
    if bits == 32:
        return tuple([torch.zeros(p.numel(), dtype=torch.float32, device=p.device) for p in params] for _ in range(2))
    if bits != 8:
        raise ValueError(f"bits: {bits}, 8 or 32 expected")
    codes = tuple([torch.zeros(p.numel(), dtype=torch.uint8, device=p.device).view(E4M3) for p in params]
                  for _ in range(2))
    scales = tuple([torch.zeros(-(-p.numel() // SCALE_BLOCK), dtype=torch.float32, device=p.device) for p in params]
                   for _ in range(2))
    return codes + scales


class AdamW:
    """A plan over the tensors of an optimizer (tg_adamw): their addresses are
    copied to the device once, a step is one launch.

    params    bfloat16, float16 or float32 tensors, all of one type
    grads     one per parameter, of the parameters' type or float32
    m, v      moments: float32, or float8_e4m3fn with m_scales and v_scales
    masters   float32 copies of 16-bit parameters (optional)

    Tensors are contiguous and of any shape; their buffers are kept, so
    gradients are written in place from step to step (set_grads takes new
    ones).  A step belongs to the stream that is current when it is called.  A
    graph that captured a step is not to be replayed after set_grads or close,
    which free the table it reads."""

    def __init__(self, params, grads, m, v, m_scales=None, v_scales=None, masters=None):
        self.tensors = dict(param=list(params), grad=list(grads), m=list(m), v=list(v))
        for name, given in (("m_scale", m_scales), ("v_scale", v_scales), ("master", masters)):
            if given is not None:
                self.tensors[name] = list(given)
        self.h = None
        self._create()

    def _create(self):
        lib = load_library()
        ts = self.tensors
        params = ts["param"]
        device = torch.cuda.current_device()
        dtype = params[0].dtype if params else torch.float32
        grad = ts["grad"][0].dtype if ts["grad"] else dtype
        state = ts["m"][0].dtype if ts["m"] else torch.float32
        if dtype not in TYPES or dtype == E4M3:
            raise ValueError(f"params: dtype {dtype}, float32, bfloat16 or float16 expected")
        if grad not in (dtype, torch.float32):
            raise ValueError(f"grads: dtype {grad}, {dtype} or float32 expected")
        if state not in (torch.float32, E4M3):
            raise ValueError(f"m: dtype {state}, float32 or float8_e4m3fn expected")
        eight = state == E4M3
        if eight != ("m_scale" in ts) or eight != ("v_scale" in ts):
            raise ValueError("m_scales and v_scales belong to moments in 8 bits")
        want = dict(param=dtype, grad=grad, m=state, v=state, m_scale=torch.float32, v_scale=torch.float32,
                    master=torch.float32)
        table = (TgAdamwTensor * len(params))()
        for name, tensors in ts.items():
            if len(tensors) != len(params):
                raise ValueError(f"{name}: {len(tensors)} tensors for {len(params)} parameters")
            for i, t in enumerate(tensors):
                n = params[i].numel()
                if name.endswith("scale"):
                    n = -(-n // SCALE_BLOCK)
                if t.get_device() != device:
                    raise _elsewhere(t, f"{name} {i}", device)
                if t.dtype != want[name]:
                    raise ValueError(f"{name} {i}: dtype {t.dtype}, {want[name]} expected")
                if not t.is_contiguous() or t.numel() != n:
                    raise ValueError(f"{name} {i}: {n} contiguous elements expected")
                setattr(table[i], name, t.data_ptr())
        for i, p in enumerate(params):
            table[i].n = p.numel()
        h = ctypes.c_void_p()
        T._check(lib.tg_adamw_create(table, len(params), TYPES[dtype], TYPES[grad], 8 if eight else 32,
                                     ctypes.byref(h)), "tg_adamw_create")
        self.close()
        self.h, self.device = h, device

    def set_grads(self, grads):
        """Takes other gradient buffers; waits for the device.  Graphs that
        captured a step before must be captured anew."""
        kept = self.tensors["grad"]
        self.tensors["grad"] = list(grads)
        try:
            self._create()
        except Exception:
            self.tensors["grad"] = kept
            raise

    def step(self, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, seed=0):
        """One step (steps count from 1).  seed: random bits for the rounding of
        8-bit moments, mixed with the step's number."""
        if self.h is None:
            raise ValueError("the plan is closed")
        rates = TgAdamwRates(lr, beta1, beta2, eps, weight_decay, grad_scale, step, seed & 0xFFFFFFFF, 0)
        T._check(load_library().tg_adamw_step(self.h, rates, _stream(self.device)), "tg_adamw_step")

    def close(self):
        if self.h is not None:
            load_library().tg_adamw_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
