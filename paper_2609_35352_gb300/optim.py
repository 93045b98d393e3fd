"""Binding of include/fiona_optim.h: AdamW over the tensors of many models at once
(argument marshalling and the state's buffers; the arithmetic is defined in the
header).

Weights and gradients are contiguous torch tensors on the context's device.  As
everywhere in this package, `stream` is a torch stream, a handle, or None for the
legacy default stream.
"""
from __future__ import annotations

import ctypes
from typing import Any, Optional, Sequence, Union

import numpy as np
import torch

from . import adapters as AD
from . import fiona as F

BLOCK = 256
FIONA_ADAMW_8BIT, FIONA_ADAMW_SKIP_NONFINITE = 1, 2

EXPORTED = ("fiona_adamw_state_count", "fiona_adamw_create", "fiona_adamw_destroy", "fiona_adamw_reset", "fiona_adamw_step",
            "fiona_adamw_moments", "fiona_adamw_load_moments")

TENSOR_DTYPE = np.dtype([("param", "<u8"), ("grad", "<u8"), ("count", "<u8"), ("dtype", "<u4"), ("group", "<u4")])
GROUP_DTYPE = np.dtype([(n, "<f8") for n in ("beta1", "beta2", "eps", "weight_decay", "max_norm")])


class State(ctypes.Structure):  # fiona_adamw_state
    _fields_ = [(n, ctypes.c_void_p) for n in ("m", "v", "m_scale", "v_scale", "master", "steps", "lr", "norms")]


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = F.lib()
        p, u32, u64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64
        L.fiona_adamw_state_count.argtypes = [u32, p, ctypes.POINTER(u64)]
        L.fiona_adamw_create.argtypes = [p, u32, p, u32, p, u32, p, ctypes.POINTER(p)]
        L.fiona_adamw_destroy.argtypes, L.fiona_adamw_destroy.restype = [p], None
        L.fiona_adamw_reset.argtypes = [p, p]
        L.fiona_adamw_step.argtypes = [p, p, p]
        L.fiona_adamw_moments.argtypes = [p, p, u32, p, p]
        L.fiona_adamw_load_moments.argtypes = [p, p, u32, p, p]
        for name in EXPORTED:
            if name != "fiona_adamw_destroy":
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _per_group(value: Any, n: int, name: str) -> np.ndarray:
    v = np.asarray(value, dtype=np.float64)
    if v.ndim > 1 or (v.ndim == 1 and v.shape[0] != n):
        raise ValueError("%s: a number, or one for each of the %d groups" % (name, n))
    return np.ascontiguousarray(np.broadcast_to(v, (n,)))


class AdamW:
    """fiona_adamw.  groups[i] is the group of params[i]: a number, or one for each
    slice along its first axis (an adapter tensor [clients][...] whose clients are
    models of their own); None: all are group 0.  lr, the two betas, eps,
    weight_decay and max_norm are numbers or one for each group (n_groups: as many as
    there are, or more).  max_norm None: norms are not taken, and `norms` is None
    (infinity: taken, not clipped).

    State, which the caller may read, save and write in stream order: `m`, `v`
    (fp32, or codes: int8 and uint8, with `m_scale` and `v_scale`), `master` (or
    None), each flat, tensor by tensor and slice by slice from multiples of 256 on
    (`places`: where each starts); `steps` [groups] int64, `lr` [groups] fp32, which
    every step reads, and `norms` [groups] fp32 of the last step.  It starts from
    zero, masters from the weights (`reset`, on the device's current stream)."""

    def __init__(self, ctx: F.Context, params: Sequence[Any], grads: Sequence[Any], groups: Optional[Sequence[Any]] = None,
                 lr: Union[float, Sequence[float]] = 1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, max_norm=None,
                 skip_nonfinite: bool = False, state_bits: int = 32, master: bool = False, n_groups: Optional[int] = None):
        self.handle = None
        if state_bits not in (8, 32):
            raise ValueError("state_bits: 8 or 32 expected")
        if len(params) != len(grads) or (groups is not None and len(groups) != len(params)):
            raise ValueError("one gradient and one group (or list of groups) for each tensor expected")
        dev, parts = AD._device(ctx) or torch.device("cpu"), []
        for i, (p, g) in enumerate(zip(params, grads)):
            if not p.is_contiguous() or p.device != dev:
                raise ValueError("params[%d]: a contiguous tensor on the context's device expected" % i)
            at = AD._whole(g, p.shape, p.dtype, dev, "grads[%d]" % i)
            of, name = 0 if groups is None else groups[i], "groups[%d]" % i
            each = np.ndim(of) > 0
            of = AD._indices(of if each else [of], np.uint32, name)
            if each and (of.ndim != 1 or p.dim() == 0 or of.shape[0] != p.shape[0]):
                raise ValueError("%s: a number, or one for each of the tensor's slices, expected" % name)
            n = p.numel() // max(of.shape[0], 1)
            step = np.arange(of.shape[0], dtype=np.uint64) * np.uint64(n * p.element_size())
            t = np.zeros(of.shape[0], TENSOR_DTYPE)
            t["param"], t["grad"] = step + np.uint64(p.data_ptr()), step + np.uint64(at)
            t["count"], t["dtype"], t["group"] = n, AD._dtype(p.dtype), of
            parts.append(t)
        tensors = np.concatenate(parts) if parts else np.zeros(0, TENSOR_DTYPE)
        most = int(tensors["group"].max()) + 1 if tensors.shape[0] else 1
        self.n_groups = n = most if n_groups is None else int(AD._indices([n_groups], np.uint32, "n_groups")[0])
        if n < most or n < 1:
            raise ValueError("n_groups: %d, but there is a group %d" % (n, most - 1))
        settings = np.zeros(n, GROUP_DTYPE)
        for name, value in (("beta1", betas[0]), ("beta2", betas[1]), ("eps", eps), ("weight_decay", weight_decay),
                            ("max_norm", np.inf if max_norm is None else max_norm)):
            settings[name] = _per_group(value, n, name)
        rate = _per_group(lr, n, "lr")
        count = ctypes.c_uint64()
        F._check(lib().fiona_adamw_state_count(tensors.shape[0], tensors.ctypes.data, ctypes.byref(count)), "fiona_adamw_state_count")
        total, bits8 = count.value, state_bits == 8
        padded = (tensors["count"] + np.uint64(BLOCK - 1)) // np.uint64(BLOCK) * np.uint64(BLOCK)
        self.places = np.cumsum(padded) - padded

        def room(k, dtype):
            return torch.empty(k, dtype=dtype, device=dev)

        self.m = room(total, torch.int8 if bits8 else torch.float32)
        self.v = room(total, torch.uint8 if bits8 else torch.float32)
        self.m_scale, self.v_scale = (room(total // BLOCK, torch.float32) if bits8 else None for _ in range(2))
        self.master = room(total, torch.float32) if master else None
        self.steps, self.lr = room(n, torch.int64), torch.from_numpy(rate.astype(np.float32)).to(dev)
        self.norms = room(n, torch.float32) if max_norm is not None or skip_nonfinite else None
        state = State(*(None if t is None else t.data_ptr() or None
                        for t in (self.m, self.v, self.m_scale, self.v_scale, self.master, self.steps, self.lr, self.norms)))
        flags = (FIONA_ADAMW_8BIT if bits8 else 0) | (FIONA_ADAMW_SKIP_NONFINITE if skip_nonfinite else 0)
        h = ctypes.c_void_p()
        F._check(lib().fiona_adamw_create(ctx.handle, tensors.shape[0], tensors.ctypes.data, n, settings.ctypes.data, flags,
                                          ctypes.byref(state), ctypes.byref(h)), "fiona_adamw_create")
        self.ctx, self.handle, self._dev = ctx, h, dev
        self._keep = (list(params), list(grads))  # (their addresses are in the optimizer)
        if dev.type == "cuda":
            self.reset(torch.cuda.current_stream(dev))

    def reset(self, stream=None) -> None:
        """fiona_adamw_reset: moments and steps zero, masters from the weights."""
        F._check(lib().fiona_adamw_reset(self.handle, AD._handle(stream)), "fiona_adamw_reset")

    def step(self, active=None, stream=None) -> None:
        """fiona_adamw_step: one step of every group, or of those where `active`
        [groups] (bool or uint8, on the device) is set."""
        at = None
        if active is not None:
            if active.dtype is not torch.bool and active.dtype is not torch.uint8:
                raise ValueError("active: bool or uint8 expected, got %s" % active.dtype)
            at = AD._whole(active, (self.n_groups,), active.dtype, self._dev, "active")
        rc = lib().fiona_adamw_step(self.handle, AD._handle(stream), at)
        if rc:
            F._check(rc, "fiona_adamw_step")

    def _values(self, m, v) -> tuple:
        dt = next((t.dtype for t in (m, v) if t is not None), torch.float32)
        at = []
        for t, name in ((m, "m"), (v, "v")):
            if t is not None and (t.numel() != self.m.numel() or t.dtype != dt or t.device != self._dev or not t.is_contiguous()):
                raise ValueError("%s: %d contiguous values of one type on the context's device expected" % (name, self.m.numel()))
            at.append(None if t is None else t.data_ptr() or None)
        return AD._dtype(dt), at[0], at[1]

    def moments(self, m=None, v=None, stream=None) -> None:
        """fiona_adamw_moments: the moments as values, into m and v (either may be None)."""
        F._check(lib().fiona_adamw_moments(self.handle, AD._handle(stream), *self._values(m, v)), "fiona_adamw_moments")

    def load_moments(self, m=None, v=None, stream=None) -> None:
        """fiona_adamw_load_moments: the moments from values, as `moments` lays them out."""
        F._check(lib().fiona_adamw_load_moments(self.handle, AD._handle(stream), *self._values(m, v)), "fiona_adamw_load_moments")

    def close(self) -> None:
        if getattr(self, "handle", None):
            lib().fiona_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
