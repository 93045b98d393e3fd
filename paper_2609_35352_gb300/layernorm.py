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


def _weights(shape: tuple, dt: Any, dev: Any, *named: tuple) -> tuple:
    """The element type of weight, bias or their gradients (that of the rows, or
    fp32, the same for all that are given) and their addresses."""
    wt, at = dt, []
    for t, _ in named:
        if t is not None:
            wt = t.dtype
            break
    if wt != dt and wt != torch.float32:
        raise ValueError("weights of %s: %s or float32 expected" % (wt, dt))
    for t, name in named:
        at.append(0 if t is None else AD._whole(t, shape, wt, dev, name))
    return AD._dtype(wt), at


def _shape(x: Any, name: str) -> tuple:
    if x.dim() != 2:
        raise ValueError("%s [rows][cols] expected" % name)
    if not 1 <= x.shape[1] <= MAX_COLS:
        raise ValueError("%s: 1 to %d columns expected" % (name, MAX_COLS))
    return x.shape


def layer_norm(ctx: F.Context, x, out, weight=None, bias=None, eps: float = 1e-5, residual=None,
               dropout: Optional[AD.Dropout] = None, sum=None, mean=None, rstd=None, stream=None) -> None:
    """fiona_layer_norm: s = residual + D(x) by rows, out = weight (s - mean) rstd +
    bias; sum gets s, mean and rstd [rows] fp32 what the gradient needs.  out may
    be x or residual, and so may sum."""
    shape = _shape(x, "x")
    dt, dev, f32 = x.dtype, AD._device(ctx), torch.float32
    rows, cols = shape
    wt, (pw, pb) = _weights((cols,), dt, dev, (weight, "weight"), (bias, "bias"))
    call = _call(rows, cols, AD._dtype(dt), wt, 0, eps, pw, pb,
                 x.data_ptr(), AD._matrix(x, shape, dt, dev, "x"),
                 *((0, 0) if residual is None else (residual.data_ptr(), AD._matrix(residual, shape, dt, dev, "residual"))),
                 out.data_ptr(), AD._matrix(out, shape, dt, dev, "out"),
                 *((0, 0) if sum is None else (sum.data_ptr(), AD._matrix(sum, shape, dt, dev, "sum"))),
                 0 if mean is None else AD._whole(mean, (rows,), f32, dev, "mean"),
                 0 if rstd is None else AD._whole(rstd, (rows,), f32, dev, "rstd")) \
        + (_no_dropout if dropout is None else dropout._spec)
    rc = lib().fiona_layer_norm(ctx.handle, AD._handle(stream), call)
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
    wt, (pw, pdw, pdb) = _weights((cols,), dt, dev, (weight, "weight"), (dweight, "dweight"), (dbias, "dbias"))

    def matrix(t, name):
        return (0, 0) if t is None else (t.data_ptr(), AD._matrix(t, shape, dt, dev, name))

    pwork, nwork = (0, 0) if work is None else (AD._workspace(work, dev), work.nbytes)
    call = _grad_call(rows, cols, AD._dtype(dt), wt, 0, pw, *matrix(dy, "dy"), *matrix(sum, "sum"),
                      AD._whole(mean, (rows,), f32, dev, "mean"), AD._whole(rstd, (rows,), f32, dev, "rstd"),
                      *matrix(dsum, "dsum"), *matrix(dx, "dx"), *matrix(dresidual, "dresidual"), pdw, pdb, pwork, nwork) \
        + (_no_dropout if dropout is None else dropout._spec)
    rc = lib().fiona_layer_norm_backward(ctx.handle, AD._handle(stream), call)
    if rc:
        F._check(rc, "fiona_layer_norm_backward")
