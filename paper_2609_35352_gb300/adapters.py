"""Binding of include/fiona_adapter.h: low-rank adapters of many requests beside
a shared projection, and dropout whose mask is never stored (argument
marshalling only; the arithmetic and the mask are defined in the header).

Tensors are torch tensors on the context's device, rows with any stride and
contiguous columns; adapter weights and their gradients are contiguous.  As
everywhere in this package, `stream` is a torch stream, a handle, or None for
the legacy default stream.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Any, Optional, Sequence

import numpy as np
import torch

from . import fiona as F

FIONA_F32, FIONA_F16, FIONA_BF16 = 0, 1, 2
MAX_RANK = 128

EXPORTED = ("fiona_adapter_batch_create", "fiona_adapter_batch_forward_only", "fiona_adapter_batch_destroy", "fiona_adapter_work_bytes",
            "fiona_adapter_forward", "fiona_adapter_backward", "fiona_dropout")


# fiona_adapter_layer and fiona_dropout_spec as bytes (a call on one token is its
# marshalling for the most part: packing takes a quarter of a ctypes structure's time)
_layer = struct.Struct("=IIIIQQ").pack
_dropout_spec = struct.Struct("=QQd").pack


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = F.lib()
        p, u32, u64, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int
        L.fiona_adapter_batch_create.argtypes = [p, u32, p, p, u32, p, p, u32, ctypes.POINTER(p)]
        L.fiona_adapter_batch_forward_only.argtypes = [p]
        L.fiona_adapter_batch_destroy.argtypes = [p]
        L.fiona_adapter_batch_destroy.restype = None
        L.fiona_adapter_work_bytes.argtypes = [p, u32, u32, u32, ctypes.POINTER(u64)]
        L.fiona_adapter_forward.argtypes = [p, p, p, p, u64, p, u64, p, u64, p, p, p, u64]
        L.fiona_adapter_backward.argtypes = [p, p, p, p, u64, p, p, u64, p, u64, p, u64, p, p, p, p, u64]
        L.fiona_dropout.argtypes = [p, p, u32, u64, u64, p, u64, p, u64, p, u64, p]
        for name in EXPORTED:
            if name != "fiona_adapter_batch_destroy":
                getattr(L, name).restype = i32
        _lib = L
    return _lib


_dtypes = {torch.float32: FIONA_F32, torch.float16: FIONA_F16, torch.bfloat16: FIONA_BF16}


def _dtype(t: Any) -> int:
    d = _dtypes.get(t)
    if d is None:
        raise ValueError("element type %s: float32, float16 or bfloat16 expected" % t)
    return d


def _refuse(t: Any, shape: tuple, dtype: Any, device: Any, name: str) -> None:
    if t.shape != shape or t.dtype != dtype:
        raise ValueError("%s: %s of %s expected, got %s of %s" % (name, shape, dtype, tuple(t.shape), t.dtype))
    if t.device != device:
        raise ValueError("%s is on %s, the context on %s" % (name, t.device, device))
    raise ValueError("%s: columns must be contiguous" % name)


def _matrix(t: Any, shape: tuple, dtype: Any, device: Any, name: str) -> int:
    """The row stride of a matrix with contiguous columns."""
    if t.shape == shape and t.dtype == dtype and t.device == device:
        row, col = t.stride()
        if col == 1 or shape[1] == 1:
            return row if shape[0] > 1 else shape[1]
    _refuse(t, shape, dtype, device, name)


def _whole(t: Any, shape: tuple, dtype: Any, device: Any, name: str) -> int:
    """The address of a contiguous tensor."""
    if t.shape == shape and t.dtype == dtype and t.device == device and t.is_contiguous():
        return t.data_ptr()
    _refuse(t, shape, dtype, device, name)


def _workspace(t: Any, device: Any) -> int:
    """The address of a workspace."""
    if t is None or t.device != device or not t.is_contiguous():
        raise ValueError("a contiguous workspace on the context's device expected (Batch.workspace)")
    return t.data_ptr()


_devices: dict = {}


def _device(ctx: F.Context) -> Any:
    """The context's device (None: validation only)."""
    d = _devices.get(ctx.device)
    if d is None and ctx.device >= 0:
        d = _devices[ctx.device] = torch.device("cuda", ctx.device)
    return d


class Dropout:
    """A dropout: probability, and the place of its mask in the generator's
    stream.  `advance` moves on past a matrix of the given size."""

    def __init__(self, p: float, seed: int, offset: int = 0):
        self.p, self.seed, self.offset = float(p), int(seed), int(offset)
        m = (1 << 64) - 1
        self._spec = _dropout_spec(self.seed & m, self.offset & m, self.p)

    def advance(self, rows: int, cols: int) -> "Dropout":
        return Dropout(self.p, self.seed, self.offset + rows * ((cols + 3) // 4))


def _handle(stream: Any) -> int:
    return 0 if stream is None else stream if type(stream) is int else stream.cuda_stream


def _indices(values: Any, dtype: Any, name: str) -> np.ndarray:
    """Whole numbers as a C array (numpy would wrap what does not fit, and cut fractions)."""
    v = np.asarray(values)
    if v.dtype == dtype or v.size == 0:
        return np.ascontiguousarray(v, dtype)
    limits, whole = np.iinfo(dtype), v.dtype.kind in "iu"
    if not (whole or v.dtype.kind == "f") or not (v.min() >= limits.min and v.max() <= (limits.max if whole else min(limits.max, 1 << 53))) \
            or not (whole or (v == np.floor(v)).all()):
        raise ValueError("%s: whole numbers from %d to %d expected" % (name, limits.min, limits.max))
    return np.ascontiguousarray(v, dtype)


class Batch:
    """fiona_adapter_batch: request r owns the rows starts[r] to starts[r + 1] and
    uses adapter adapters[r] (-1: none); adapter a has rank ranks[a] and scale
    scales[a] (None: 1).  One batch serves every layer of a model.  One without
    `gradients` is for forward calls only, and its workspaces are smaller."""

    def __init__(self, ctx: F.Context, starts: Sequence[int], adapters: Sequence[int], ranks: Sequence[int],
                 r_max: int, scales: Optional[Sequence[float]] = None, gradients: bool = True):
        s, a, r = (_indices(v, t, n) for v, t, n in ((starts, np.uint64, "starts"), (adapters, np.int32, "adapters"),
                                                     (ranks, np.uint32, "ranks")))
        r_max = r_max if type(r_max) is int and 0 <= r_max < 1 << 32 else int(_indices([r_max], np.uint32, "r_max")[0])
        if s.ndim != 1 or a.ndim != 1 or r.ndim != 1 or s.shape[0] != a.shape[0] + 1:
            raise ValueError("starts must have one entry more than adapters")
        c = None
        if scales is not None:
            c = np.ascontiguousarray(np.asarray(scales, dtype=np.float32))
            if c.shape != r.shape:
                raise ValueError("one scale per adapter expected")
        h = ctypes.c_void_p()
        F._check(lib().fiona_adapter_batch_create(ctx.handle, a.shape[0], s.ctypes.data, a.ctypes.data, r.shape[0],
                                                  r.ctypes.data, None if c is None else c.ctypes.data, r_max,
                                                  ctypes.byref(h)), "fiona_adapter_batch_create")
        self.ctx, self.handle = ctx, h
        if not gradients:
            F._check(lib().fiona_adapter_batch_forward_only(h), "fiona_adapter_batch_forward_only")
        self.n_tokens, self.n_adapters, self.r_max = int(s[-1]), int(r.shape[0]), r_max
        self._dev = _device(ctx)

    def work_bytes(self, d_in: int, d_out: int, dtype: Any) -> int:
        n = ctypes.c_uint64()
        F._check(lib().fiona_adapter_work_bytes(self.handle, int(d_in), int(d_out), _dtype(dtype), ctypes.byref(n)),
                 "fiona_adapter_work_bytes")
        return n.value

    def workspace(self, d_in: int, d_out: int, dtype: Any):
        """A workspace for calls on layers of these sizes;
        calls that may overlap in time need one each."""
        return torch.empty(max(self.work_bytes(d_in, d_out, dtype), 16), dtype=torch.uint8,
                           device="cuda:%d" % self.ctx.device)

    def _layer(self, x, A, B):
        if x.dim() != 2 or B.dim() != 3:
            raise ValueError("x [tokens][d_in] and B [adapters][d_out][r_max] expected")
        d_in, d_out, dev = x.shape[1], B.shape[1], self._dev
        dt = x.dtype
        return d_in, d_out, _layer(d_in, d_out, _dtype(dt), 0,
                                   _whole(A, (self.n_adapters, self.r_max, d_in), dt, dev, "A"),
                                   _whole(B, (self.n_adapters, d_out, self.r_max), dt, dev, "B"))

    def forward(self, x, A, B, out, base=None, h=None, dropout: Optional[Dropout] = None, work=None,
                stream=None) -> None:
        """fiona_adapter_forward: out = base + s_a (D(x) A_a^T) B_a^T by rows;
        h [tokens][r_max] fp32, where given, gets D(x) A_a^T."""
        d_in, d_out, layer = self._layer(x, A, B)
        T, dt, dev = self.n_tokens, x.dtype, self._dev
        ldx = _matrix(x, (T, d_in), dt, dev, "x")
        ld_out = _matrix(out, (T, d_out), dt, dev, "out")
        ld_base, p_base = (0, None) if base is None else (_matrix(base, (T, d_out), dt, dev, "base"), base.data_ptr())
        ph = None if h is None else _whole(h, (T, self.r_max), torch.float32, dev, "h")
        p_work = _workspace(work, dev)
        rc = lib().fiona_adapter_forward(self.handle, _handle(stream), layer, x.data_ptr(), ldx, p_base, ld_base,
                                         out.data_ptr(), ld_out, ph, None if dropout is None else dropout._spec,
                                         p_work, work.nbytes)
        if rc:
            F._check(rc, "fiona_adapter_forward")

    def backward(self, x, h, dy, A, B, dx, dA, dB, dx_base=None, dropout: Optional[Dropout] = None, work=None,
                 stream=None) -> None:
        """fiona_adapter_backward: dx, dA and dB (overwritten) from the x, h and
        dropout of the forward pass and the gradient dy of its out."""
        d_in, d_out, layer = self._layer(x, A, B)
        T, dt, dev = self.n_tokens, x.dtype, self._dev
        ldx = _matrix(x, (T, d_in), dt, dev, "x")
        ld_dy = _matrix(dy, (T, d_out), dt, dev, "dy")
        ld_dx = _matrix(dx, (T, d_in), dt, dev, "dx")
        ld_base, p_base = (0, None) if dx_base is None else (_matrix(dx_base, (T, d_in), dt, dev, "dx_base"), dx_base.data_ptr())
        ph = _whole(h, (T, self.r_max), torch.float32, dev, "h")
        pA = _whole(dA, A.shape, dt, dev, "dA")
        pB = _whole(dB, B.shape, dt, dev, "dB")
        p_work = _workspace(work, dev)
        rc = lib().fiona_adapter_backward(self.handle, _handle(stream), layer, x.data_ptr(), ldx, ph, dy.data_ptr(),
                                          ld_dy, p_base, ld_base, dx.data_ptr(), ld_dx, pA, pB,
                                          None if dropout is None else dropout._spec, p_work, work.nbytes)
        if rc:
            F._check(rc, "fiona_adapter_backward")

    def close(self) -> None:
        if getattr(self, "handle", None):
            lib().fiona_adapter_batch_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def dropout(ctx: F.Context, x, out, drop: Dropout, residual=None, stream=None) -> None:
    """fiona_dropout: out = residual + D(x) on matrices [rows][cols] (out may be
    x or residual)."""
    if x.dim() != 2:
        raise ValueError("x [rows][cols] expected")
    shape, dt, dev = x.shape, x.dtype, _device(ctx)
    ldx = _matrix(x, shape, dt, dev, "x")
    ld_out = _matrix(out, shape, dt, dev, "out")
    ld_res = 0 if residual is None else _matrix(residual, shape, dt, dev, "residual")
    rc = lib().fiona_dropout(ctx.handle, _handle(stream), _dtype(dt), shape[0], shape[1], x.data_ptr(), ldx,
                             None if residual is None else residual.data_ptr(), ld_res, out.data_ptr(), ld_out, drop._spec)
    if rc:
        F._check(rc, "fiona_dropout")


def dropout_backward(ctx: F.Context, dy, dx, drop: Dropout, stream=None) -> None:
    """The gradient of x through `dropout`: the same mask and factor on dy (the
    residual's gradient is dy itself)."""
    dropout(ctx, dy, dx, drop, stream=stream)
