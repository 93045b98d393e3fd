"""The layer norm's entry points on the host (no GPU): exports, refusals, workspace
sizes, and what the binding checks before it passes addresses on."""
import ctypes
import os
import re
import struct

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_35352_gb300 import adapters as AD
from paper_2609_35352_gb300 import build as B
from paper_2609_35352_gb300 import fiona as F
from paper_2609_35352_gb300 import layernorm as LN
from paper_2609_35352_gb300 import workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, NODEVICE = F.FIONA_ERR_ARG, F.FIONA_ERR_NODEVICE
P, U32, U64, F64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_double


class Spec(ctypes.Structure):
    _fields_ = [("seed", U64), ("offset", U64), ("p", F64)]


class Call(ctypes.Structure):  # fiona_layer_norm_call
    _fields_ = [("rows", U64), ("cols", U32), ("dtype", U32), ("weight_dtype", U32), ("reserved", U32), ("eps", F64), ("weight", P),
                ("bias", P), ("x", P), ("ldx", U64), ("residual", P), ("ld_residual", U64), ("out", P), ("ld_out", U64), ("sum", P),
                ("ld_sum", U64), ("mean", P), ("rstd", P), ("drop", Spec)]


class GradCall(ctypes.Structure):  # fiona_layer_norm_grad_call
    _fields_ = [("rows", U64), ("cols", U32), ("dtype", U32), ("weight_dtype", U32), ("reserved", U32), ("weight", P), ("dy", P),
                ("ld_dy", U64), ("sum", P), ("ld_sum", U64), ("mean", P), ("rstd", P), ("dsum", P), ("ld_dsum", U64), ("dx", P),
                ("ld_dx", U64), ("dresidual", P), ("ld_dresidual", U64), ("dweight", P), ("dbias", P), ("work", P), ("work_bytes", U64),
                ("drop", Spec)]


@pytest.fixture(scope="module")
def ctx():
    B.build()
    return F.Context(1024, W.ntt_primes(1024, 40, 1), device=F.FIONA_DEVICE_NONE)


def test_exports(ctx):
    text = open(os.path.join(ROOT, "include", "fiona_norm.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(fiona_\w+)\s*\(", text)))
    assert names == sorted(LN.EXPORTED)
    for n in names:
        assert hasattr(ctypes.CDLL(F.LIB_PATH), n)


def test_packed_structures():
    """The binding's packed arguments are the header's structures."""
    v = list(range(1, 19))
    v[5] = 0.5
    assert LN._call(*v) + AD.Dropout(0.25, 3, 4)._spec == bytes(Call(*v, Spec(3, 4, 0.25)))
    v = list(range(1, 23))
    assert LN._grad_call(*v) + AD.Dropout(0.25, 3, 4)._spec == bytes(GradCall(*v, Spec(3, 4, 0.25)))
    assert len(struct.pack("=QQd", 0, 0, 0.0)) == ctypes.sizeof(Spec)


ROWS, COLS = 6, 40


class Case:
    """A call on host memory of the right sizes: everything is checked, nothing runs
    (the context has no device)."""

    def __init__(self, ctx, backward, dtype=2, weight_dtype=2):
        self.ctx, self.backward = ctx, backward
        n = ROWS * COLS * 4 + 64
        size = ctypes.c_uint64()
        assert LN.lib().fiona_layer_norm_work_bytes(ctx.handle, ROWS, COLS, ctypes.byref(size)) == 0
        self.keep = {}
        self.c = GradCall() if backward else Call()
        c = self.c
        c.rows, c.cols, c.dtype, c.weight_dtype, c.drop = ROWS, COLS, dtype, weight_dtype, Spec(1, 2, 0.5)
        for name, kind in c._fields_:
            if kind is P:
                b = self.keep[name] = np.zeros(size.value + 64 if name == "work" else n, np.uint8)
                setattr(c, name, (b.ctypes.data + 15) // 16 * 16)
            elif name.startswith("ld"):
                setattr(c, name, COLS)
        if backward:
            c.work_bytes = size.value
        else:
            c.eps = 1e-5

    def __call__(self, c=None):
        f = LN.lib().fiona_layer_norm_backward if self.backward else LN.lib().fiona_layer_norm
        return f(self.ctx.handle, None, ctypes.byref(self.c))

    def put(self, **values):
        for k, v in values.items():
            setattr(self.c, k, v)
        return self()


FORWARD_MATRICES, BACKWARD_MATRICES = ("x", "residual", "out", "sum"), ("dy", "sum", "dsum", "dx", "dresidual")


@pytest.mark.parametrize("backward", [False, True])
def test_refused(ctx, backward):
    assert Case(ctx, backward)() == NODEVICE  # all is well but for the device
    matrices = BACKWARD_MATRICES if backward else FORWARD_MATRICES
    outputs = ("dx", "dresidual") if backward else ("out", "sum")
    vectors = ("weight", "dweight", "dbias") if backward else ("weight", "bias")
    for k in ("dy", "sum", "mean", "rstd", "work") if backward else ("x", "out"):
        c = Case(ctx, backward)
        assert c.put(**{k: None}) == ARG, k
        assert F.last_error()
    for k in matrices + vectors:
        c = Case(ctx, backward)
        assert c.put(**{k: getattr(c.c, k) + 1}) == ARG, k
    for k in ("mean", "rstd"):
        c = Case(ctx, backward)
        assert c.put(**{k: getattr(c.c, k) + 2}) == ARG, k
    for k in outputs:
        assert Case(ctx, backward).put(**{"ld_" + k: COLS - 1}) == ARG, k
    for k in matrices:
        assert Case(ctx, backward).put(**{"ldx" if k == "x" else "ld_" + k: 1 << 40}) == ARG, k
    for p in (-0.1, 1.5, float("nan")):
        assert Case(ctx, backward).put(drop=Spec(1, 2, p)) == ARG
    for field, value in (("rows", 1 << 40), ("cols", 0), ("cols", (1 << 20) + 1), ("dtype", 3), ("weight_dtype", 1), ("reserved", 1)):
        assert Case(ctx, backward).put(**{field: value}) == ARG, field
    if backward:
        c = Case(ctx, backward)
        assert c.put(work_bytes=c.c.work_bytes - 1) == ARG
        assert Case(ctx, backward).put(work=c.c.work + 8) == ARG
        assert Case(ctx, backward).put(dx=None, dresidual=None, dweight=None, dbias=None) == ARG
    else:
        for eps in (-1e-9, 1e-39, 5e-324, float("nan"), float("inf")):
            assert Case(ctx, backward).put(eps=eps) == ARG
        for eps in (0.0, 2.0 ** -126):
            assert Case(ctx, backward).put(eps=eps) == NODEVICE
    assert (LN.lib().fiona_layer_norm_backward if backward else LN.lib().fiona_layer_norm)(ctx.handle, None, None) == ARG


@pytest.mark.parametrize("backward", [False, True])
def test_overlaps(ctx, backward):
    """Every output against every other buffer: refused but where the header allows it."""
    allowed = {"dx": ("dy", "sum", "dsum"), "dresidual": ("dy", "sum", "dsum"), "out": ("x", "residual"), "sum": ("x", "residual")}
    outputs = ("dx", "dresidual", "dweight", "dbias", "work") if backward else ("out", "sum", "mean", "rstd")
    pointers = [n for n, kind in (GradCall if backward else Call)._fields_ if kind is P]
    for o in outputs:
        for k in pointers:
            if o == k:
                continue
            c = Case(ctx, backward)
            fine = k in allowed.get(o, ()) or (o in allowed.get(k, ()) and backward and o in ("sum",))
            assert c.put(**{o: getattr(c.c, k)}) == (NODEVICE if fine else ARG), (o, k)
            if fine:  # the same place, but not the same matrix
                c = Case(ctx, backward)
                assert c.put(**{o: getattr(c.c, k) + 16}) == ARG, (o, k)
                c = Case(ctx, backward)
                assert c.put(**{o: getattr(c.c, k), "ld_" + o: COLS + 8}) == ARG, (o, k)


def test_accepted(ctx):
    for k in ("residual", "sum", "mean", "rstd", "weight", "bias"):
        assert Case(ctx, False).put(**{k: None}) == NODEVICE, k
    for k in ("weight", "dsum", "dx", "dresidual", "dweight", "dbias"):
        assert Case(ctx, True).put(**{k: None}) == NODEVICE, k
    assert Case(ctx, True).put(dweight=None, dbias=None, work=None, work_bytes=0) == NODEVICE  # no sums: no workspace
    assert Case(ctx, False).put(ldx=0) == NODEVICE  # one row for all
    assert Case(ctx, False).put(rows=0, x=None, out=None) == F.FIONA_OK
    for dt in (0, 1, 2):
        for back in (False, True):
            assert Case(ctx, back, dt, 0)() == NODEVICE


def test_work_bytes(ctx):
    n = ctypes.c_uint64()
    L = LN.lib()
    for rows, cols in ((1, 0), (1, (1 << 20) + 1), (1 << 40, 8)):
        assert L.fiona_layer_norm_work_bytes(ctx.handle, rows, cols, ctypes.byref(n)) == ARG
    assert L.fiona_layer_norm_work_bytes(ctx.handle, 4, 8, None) == ARG
    assert L.fiona_layer_norm_work_bytes(None, 4, 8, ctypes.byref(n)) == ARG
    # one size serves any number of rows up to the one asked for
    for cols in (1, 8, 33, 768, 4096, 8192, 16384, 16385, 30000, 1 << 20):
        last = 0
        for rows in list(range(0, 40)) + [64, 100, 151, 152, 153, 303, 304, 305, 512, 1000, 1500, 4095, 4096, 16384, 100000, 155648, 155649, 1 << 22]:
            b = LN.work_bytes(ctx, rows, cols)
            assert b >= last, (rows, cols)
            last = b


def test_binding(ctx, monkeypatch):
    monkeypatch.setattr(AD, "_device", lambda c: torch.device("cpu"))

    def aligned(*shape, dtype=torch.bfloat16):
        t = torch.zeros(shape, dtype=dtype)
        assert t.data_ptr() % 16 == 0
        return t

    x, out, w = aligned(6, 40), aligned(6, 40), aligned(40)
    f = aligned(6, dtype=torch.float32)
    work = aligned(LN.work_bytes(ctx, 6, 40), dtype=torch.uint8)
    for wt in (torch.bfloat16, torch.float32):
        with pytest.raises(F.FionaError) as e:
            LN.layer_norm(ctx, x, out, weight=w.to(wt), bias=aligned(40, dtype=wt), mean=f, rstd=aligned(6, dtype=torch.float32))
        assert e.value.status == NODEVICE
        with pytest.raises(F.FionaError) as e:
            LN.layer_norm_backward(ctx, x, out, f, f, dx=aligned(6, 40), weight=w.to(wt), dweight=aligned(40, dtype=wt), work=work)
        assert e.value.status == NODEVICE
    for bad in (dict(weight=w.half()), dict(weight=w, bias=aligned(40, dtype=torch.float32)), dict(weight=aligned(41)), dict(residual=aligned(6, 41)),
                dict(residual=aligned(6, 40, dtype=torch.float16)), dict(mean=aligned(6)), dict(rstd=aligned(7, dtype=torch.float32)),
                dict(sum=aligned(40, 6).t()), dict(weight=aligned(80)[::2])):
        with pytest.raises(ValueError):
            LN.layer_norm(ctx, x, out, **bad)
    with pytest.raises(ValueError):
        LN.layer_norm(ctx, aligned(6), aligned(6))
    with pytest.raises(ValueError):
        LN.layer_norm(ctx, aligned(6, 0), aligned(6, 0))
    with pytest.raises(ValueError):
        LN.layer_norm(ctx, x.to(torch.float64), out.to(torch.float64))
    for bad in (dict(work=None), dict(work=aligned(work.numel() * 2, dtype=torch.uint8)[::2]), dict(work=work, dx=aligned(5, 40)),
                dict(work=work, dsum=aligned(6, 40, dtype=torch.float16))):
        with pytest.raises((ValueError, F.FionaError)):
            LN.layer_norm_backward(ctx, x, out, f, f, **{"dweight": aligned(40), **bad})


def test_eps_of_fp32(ctx):
    """An eps that fp32 holds, and none that it would take for infinite."""
    most = float(np.finfo(np.float32).max)
    for eps in (1.0, 1e30, most, 2.0 ** -126):
        assert Case(ctx, False).put(eps=eps) == NODEVICE, eps
    for eps in (2.0 ** 128, 1e39, 1e300):
        assert Case(ctx, False).put(eps=eps) == ARG, eps


def test_workspace_of_very_many_rows(ctx):
    """dx alone needs no workspace for fewer than 2^31 rows of up to 16384 columns; from there on
    it needs what work_bytes says.  (Addresses are made up: they are checked, and nothing runs.)"""
    for rows, cols, none in (((1 << 31) - 1, 8, True), (1 << 31, 8, False), (1 << 32, 1, False), (3, 16384, True), (3, 16385, False)):
        c = Case(ctx, True)
        c.put(rows=rows, cols=cols, dweight=None, dbias=None, dresidual=None, dsum=None, work=None, work_bytes=0)
        for i, k in enumerate(("weight", "dy", "sum", "mean", "rstd", "dx")):
            setattr(c.c, k, (i + 1) << 44)
        for k in ("dy", "sum", "dx"):
            setattr(c.c, "ldx" if k == "x" else "ld_" + k, cols)
        assert c() == (NODEVICE if none else ARG), (rows, cols)
        if not none:
            assert "workspace" in F.last_error()
            assert c.put(work=7 << 44, work_bytes=LN.work_bytes(ctx, rows, cols)) == NODEVICE
