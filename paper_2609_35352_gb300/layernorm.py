"""Binding of include/fiona_norm.h: layer norm by rows with the dropout and the
residual before it, and its gradient (argument marshalling only; the arithmetic
is defined in the header).

Tensors are torch tensors on the context's device, matrices [rows][cols] with any
row stride and contiguous columns; weight, bias, their gradients, mean and rstd
are contiguous.  As everywhere in this package, `stream` is a torch stream, a
handle, or None for the legacy default stream.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Any, Optional

import torch

from . import adapters as AD
from . import fiona as F

MAX_COLS = 1 << 20

EXPORTED = ("fiona_layer_norm", "fiona_layer_norm_backward", "fiona_layer_norm_work_bytes")

# fiona_layer_norm_call and fiona_layer_norm_grad_call, up to their fiona_dropout_spec
_call = struct.Struct("=QIIIId" + "QQ" + "QQ" * 4 + "QQ").pack
_grad_call = struct.Struct("=QIIIIQ" + "QQ" * 2 + "QQ" + "QQ" * 3 + "QQ" + "QQ").pack
_no_dropout = AD._dropout_spec(0, 0, 0.0)

_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = F.lib()
        p, u64 = ctypes.c_void_p, ctypes.c_uint64
        L.fiona_layer_norm.argtypes = [p, p, p]
        L.fiona_layer_norm_backward.argtypes = [p, p, p]
        L.fiona_layer_norm_work_bytes.argtypes = [p, u64, u64, ctypes.POINTER(u64)]
        for name in EXPORTED:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def work_bytes(ctx: F.Context, rows: int, cols: int) -> int:
    n = ctypes.c_uint64()
    F._check(lib().fiona_layer_norm_work_bytes(ctx.handle, int(rows), int(cols), ctypes.byref(n)), "fiona_layer_norm_work_bytes")
    return n.value


def workspace(ctx: F.Context, rows: int, cols: int):
    """A workspace for backward calls on matrices of up to this many rows and of
    this width; calls that may overlap in time need one each."""
    return torch.empty(max(work_bytes(ctx, rows, cols), 16), dtype=torch.uint8, device="cuda:%d" % ctx.device)


def _weight_type(dt: Any, first: Any) -> Any:
    """The element type of weight, bias and their gradients: that of the rows, or fp32."""
    if first is None or first.dtype is dt:
        return dt
    if first.dtype is not torch.float32:
        raise ValueError("weights of %s: %s or float32 expected" % (first.dtype, dt))
    return torch.float32


def _vector(t: Any, shape: tuple, dt: Any, dev: Any, name: str) -> int:
    return 0 if t is None else AD._whole(t, shape, dt, dev, name)


def _rows(t: Any, shape: tuple, dt: Any, dev: Any, name: str) -> tuple:
    """Address and row stride of a matrix (or of none)."""
    if t is None:
        return 0, 0
    if t.dtype is dt and t.shape == shape and t.device == dev:
        row, col = t.stride()
        if col == 1 or shape[1] == 1:
            return t.data_ptr(), row if shape[0] > 1 else shape[1]
    AD._refuse(t, shape, dt, dev, name)


def _shape(x: Any, name: str) -> tuple:
    if x.dim() != 2:
        raise ValueError("%s [rows][cols] expected" % name)
    shape = x.shape
    if not 1 <= shape[1] <= MAX_COLS:
        raise ValueError("%s: 1 to %d columns expected" % (name, MAX_COLS))
    return shape


def layer_norm(ctx: F.Context, x, out, weight=None, bias=None, eps: float = 1e-5, residual=None,
               dropout: Optional[AD.Dropout] = None, sum=None, mean=None, rstd=None, stream=None) -> None:
    """fiona_layer_norm: s = residual + D(x) by rows, out = weight (s - mean) rstd +
    bias; sum gets s, mean and rstd [rows] fp32 what the gradient needs.  out may
    be x or residual, and so may sum."""
    shape = _shape(x, "x")
    dt, dev, f32 = x.dtype, AD._device(ctx), torch.float32
    rows, cols = shape
    wt, per_col, per_row = _weight_type(dt, bias if weight is None else weight), (cols,), (rows,)
    px, ldx = _rows(x, shape, dt, dev, "x")
    pr, ldr = _rows(residual, shape, dt, dev, "residual")
    po, ldo = _rows(out, shape, dt, dev, "out")
    ps, lds = _rows(sum, shape, dt, dev, "sum")
    call = _call(rows, cols, AD._dtype(dt), AD._dtype(wt), 0, eps, _vector(weight, per_col, wt, dev, "weight"),
                 _vector(bias, per_col, wt, dev, "bias"), px, ldx, pr, ldr, po, ldo, ps, lds, _vector(mean, per_row, f32, dev, "mean"),
                 _vector(rstd, per_row, f32, dev, "rstd")) + (_no_dropout if dropout is None else dropout._spec)
    rc = (_lib or lib()).fiona_layer_norm(ctx.handle, AD._handle(stream), call)
    if rc:
        F._check(rc, "fiona_layer_norm")


def layer_norm_backward(ctx: F.Context, dy, sum, mean, rstd, dx=None, weight=None, dsum=None,
                        dropout: Optional[AD.Dropout] = None, dresidual=None, dweight=None, dbias=None, work=None,
                        stream=None) -> None:
    """fiona_layer_norm_backward: from the sum, mean, rstd and dropout of the forward
    pass, the gradient dy of its out and dsum of its sum: dresidual, dx (through the
    dropout), dweight and dbias, each where it is given.  dx and dresidual may each
    be dy, sum or dsum."""
    shape = _shape(dy, "dy")
    dt, dev, f32 = dy.dtype, AD._device(ctx), torch.float32
    rows, cols = shape
    wt, per_col, per_row = _weight_type(dt, next((t for t in (weight, dweight, dbias) if t is not None), None)), (cols,), (rows,)
    pw, nw = (0, 0) if work is None else (AD._workspace(work, dev), work.nbytes)
    py, ldy = _rows(dy, shape, dt, dev, "dy")
    ps, lds = _rows(sum, shape, dt, dev, "sum")
    pd, ldd = _rows(dsum, shape, dt, dev, "dsum")
    px, ldx = _rows(dx, shape, dt, dev, "dx")
    pr, ldr = _rows(dresidual, shape, dt, dev, "dresidual")
    call = _grad_call(rows, cols, AD._dtype(dt), AD._dtype(wt), 0, _vector(weight, per_col, wt, dev, "weight"), py, ldy, ps, lds,
                      AD._whole(mean, per_row, f32, dev, "mean"), AD._whole(rstd, per_row, f32, dev, "rstd"), pd, ldd, px, ldx, pr, ldr,
                      _vector(dweight, per_col, wt, dev, "dweight"), _vector(dbias, per_col, wt, dev, "dbias"), pw, nw) \
        + (_no_dropout if dropout is None else dropout._spec)
    rc = (_lib or lib()).fiona_layer_norm_backward(ctx.handle, AD._handle(stream), call)
    if rc:
        F._check(rc, "fiona_layer_norm_backward")
