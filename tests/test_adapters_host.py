"""The adapters' and the dropout's entry points on the host (no GPU): exports,
refusals, workspace sizes, and the mask's definition."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_2609_35352_gb300 import adapters as AD
from paper_2609_35352_gb300 import build as B
from paper_2609_35352_gb300 import fiona as F
from paper_2609_35352_gb300 import workloads as W

from adapter_util import keep_mask

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, PLAN, NODEVICE = F.FIONA_ERR_ARG, F.FIONA_ERR_PLAN, F.FIONA_ERR_NODEVICE


@pytest.fixture(scope="module")
def ctx():
    B.build()
    return F.Context(1024, W.ntt_primes(1024, 40, 1), device=F.FIONA_DEVICE_NONE)


class Layer(ctypes.Structure):  # fiona_adapter_layer
    _fields_ = [("d_in", ctypes.c_uint32), ("d_out", ctypes.c_uint32), ("dtype", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p)]


class DropoutSpec(ctypes.Structure):  # fiona_dropout_spec
    _fields_ = [("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("p", ctypes.c_double)]


def test_packed_structures():
    """The binding's packed arguments are the header's structures."""
    assert AD._layer(3, 5, 2, 0, 1 << 40, 7) == bytes(Layer(3, 5, 2, 0, 1 << 40, 7))
    assert AD.Dropout(0.25, -1, 1 << 63)._spec == bytes(DropoutSpec((1 << 64) - 1, 1 << 63, 0.25))


def test_exports(ctx):
    text = open(os.path.join(ROOT, "include", "fiona_adapter.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(fiona_\w+)\s*\(", text)))
    assert names == sorted(AD.EXPORTED)
    for n in names:
        assert hasattr(ctypes.CDLL(F.LIB_PATH), n)


@pytest.mark.parametrize("starts,ids,ranks,r_max,code", [
    ([0, 4, 3], [0, 0], [8], 8, PLAN),             # a request that ends before it starts
    ([1, 4], [0], [8], 8, PLAN),                   # rows that nobody owns
    ([0, 4], [1], [8], 8, PLAN),                   # no such adapter
    ([0, 4], [-2], [8], 8, PLAN),
    ([0, 4], [0], [9], 8, PLAN),                   # rank above r_max
    ([0, (1 << 26) + 1], [0], [8], 8, PLAN),       # too many rows
    ([0, 4], [0], [8], 0, ARG),
    ([0, 4], [0], [8], 129, ARG),
])
def test_batches_refused(ctx, starts, ids, ranks, r_max, code):
    with pytest.raises(F.FionaError) as e:
        AD.Batch(ctx, starts, ids, ranks, r_max)
    assert e.value.status == code


def test_null_arguments(ctx):
    L, h = AD.lib(), ctypes.c_void_p()
    s = np.array([0, 1], np.uint64)
    assert L.fiona_adapter_batch_create(None, 1, s.ctypes.data, s.ctypes.data, 0, None, None, 8,
                                        ctypes.byref(h)) == ARG
    assert L.fiona_adapter_batch_create(ctx.handle, 1, None, s.ctypes.data, 0, None, None, 8, ctypes.byref(h)) == ARG
    assert L.fiona_adapter_batch_create(ctx.handle, 1, s.ctypes.data, s.ctypes.data, 0, None, None, 8, None) == ARG
    assert not h.value
    L.fiona_adapter_batch_destroy(None)
    b = AD.Batch(ctx, [0, 3], [0], [4], 4)
    assert L.fiona_adapter_work_bytes(b.handle, 8, 8, 2, None) == ARG
    n = ctypes.c_uint64()
    for d_in, d_out, dt in ((0, 8, 2), (8, 0, 2), ((1 << 20) + 1, 8, 2), (8, 8, 3)):
        assert L.fiona_adapter_work_bytes(b.handle, d_in, d_out, dt, ctypes.byref(n)) == ARG


class Call:
    """A forward or backward call on host memory of the right sizes: everything
    is checked, nothing runs (the context has no device)."""

    def __init__(self, ctx, backward, T=6, d_in=16, d_out=24, r=8, esize=2):
        self.b, self.back = AD.Batch(ctx, [0, T], [0], [r], r), backward
        self.keep = {}
        n = {"x": T * d_in, "base": T * d_out, "out": T * d_out, "h": 2 * T * r, "dy": T * d_out, "dx_base": T * d_in,
             "dx": T * d_in, "A": r * d_in, "B": r * d_out, "dA": r * d_in, "dB": r * d_out}
        for k, v in n.items():
            self.keep[k] = np.zeros(v * esize + 64, np.uint8)
        size = self.b.work_bytes(d_in, d_out, __import__("torch").bfloat16)
        self.keep["work"] = np.zeros(size + 64, np.uint8)
        self.p = {k: (v.ctypes.data + 15) // 16 * 16 for k, v in self.keep.items()}
        self.ld = {"x": d_in, "base": d_out, "out": d_out, "dy": d_out, "dx_base": d_in, "dx": d_in}
        self.work_bytes = size
        self.layer = Layer(d_in, d_out, 2, 0, 0, 0)
        self.spec = DropoutSpec(1, 2, 0.5)

    def __call__(self):
        p, ld = self.p, self.ld
        self.layer.A, self.layer.B = p["A"], p["B"]
        L, layer, spec = AD.lib(), ctypes.byref(self.layer), ctypes.byref(self.spec)
        if self.back:
            return L.fiona_adapter_backward(self.b.handle, None, layer, p["x"], ld["x"], p["h"], p["dy"], ld["dy"],
                                            p["dx_base"], ld["dx_base"], p["dx"], ld["dx"], p["dA"], p["dB"], spec,
                                            p["work"], self.work_bytes)
        return L.fiona_adapter_forward(self.b.handle, None, layer, p["x"], ld["x"], p["base"], ld["base"], p["out"],
                                       ld["out"], p["h"], spec, p["work"], self.work_bytes)


@pytest.mark.parametrize("backward", [False, True])
def test_calls_refused(ctx, backward):
    assert Call(ctx, backward)() == NODEVICE  # all is well but for the device
    out, base = ("dx", "dx_base") if backward else ("out", "base")
    for k in ("x", out, "A", "B", "work") + (("h", "dy", "dA", "dB") if backward else ()):
        c = Call(ctx, backward)
        c.p[k] = None
        assert c() == ARG, k
        assert F.last_error()
    for k in ("x", out, base):
        c = Call(ctx, backward)
        c.p[k] += 1
        assert c() == ARG, k
    for k in ("A", "B", "h", "work") + (("dA", "dB") if backward else ()):
        c = Call(ctx, backward)
        c.p[k] += 8
        assert c() == ARG, k
    for k in ("x", "A", "B", "h", "work") + (("dy", "dA", "dB") if backward else ()):
        c = Call(ctx, backward)
        c.p[out] = c.p[k]
        assert c() == ARG, k
    c = Call(ctx, backward)
    c.ld[out] -= 1
    assert c() == ARG
    c = Call(ctx, backward)
    c.work_bytes -= 1
    assert c() == ARG
    c = Call(ctx, backward)
    c.ld["x"] = 1 << 40
    assert c() == ARG
    for p in (-0.1, 1.5, float("nan")):
        c = Call(ctx, backward)
        c.spec.p = p
        assert c() == ARG
    for field, value in (("d_in", 0), ("d_out", (1 << 20) + 1), ("dtype", 3), ("reserved", 1)):
        c = Call(ctx, backward)
        setattr(c.layer, field, value)
        assert c() == ARG, field


@pytest.mark.parametrize("backward", [False, True])
def test_calls_accepted(ctx, backward):
    out, base = ("dx", "dx_base") if backward else ("out", "base")
    c = Call(ctx, backward)
    c.p[base] = None
    assert c() == NODEVICE
    c = Call(ctx, backward)
    c.p[out] = c.p[base]  # in place
    assert c() == NODEVICE
    c = Call(ctx, backward)
    c.ld["x"] = 0  # one row for all
    assert c() == NODEVICE


def test_interleaved_columns(ctx):
    """Two column ranges of one buffer do not overlap; with other strides that is
    not said."""
    c = Call(ctx, False)
    wide = np.zeros(6 * 64 * 2 + 64, np.uint8)
    at = (wide.ctypes.data + 15) // 16 * 16
    c.p["out"], c.p["x"] = at, at + 24 * 2
    c.ld["out"] = c.ld["x"] = 64
    assert c() == NODEVICE
    c.p["x"] = at + 23 * 2
    assert c() == ARG
    c.p["x"], c.ld["x"] = at + 24 * 2, 32
    assert c() == ARG


def test_dropout_refused(ctx):
    L = AD.lib()
    buf = np.zeros(4096, np.uint8)
    at = (buf.ctypes.data + 15) // 16 * 16
    spec = DropoutSpec(1, 2, 0.5)

    def call(dtype=2, rows=4, cols=8, x=at, ldx=8, res=None, ldr=0, out=at + 1024, ldo=8, s=spec, c=ctx.handle):
        return L.fiona_dropout(c, None, dtype, rows, cols, x, ldx, res, ldr, out, ldo, None if s is None else ctypes.byref(s))

    assert call() == NODEVICE
    assert call(out=at) == NODEVICE and call(res=at + 1024, ldr=8) == NODEVICE
    assert call(rows=0) == F.FIONA_OK
    bad = [dict(dtype=3), dict(cols=0), dict(x=None), dict(out=None), dict(x=at + 1), dict(ldo=7), dict(out=at + 16),
           dict(res=at + 1024 + 16, ldr=8), dict(s=None), dict(c=None), dict(rows=1 << 40), dict(out=at, ldo=9),
           dict(s=DropoutSpec(1, 2, float("nan"))), dict(s=DropoutSpec(1, 2, -1.0))]
    for b in bad:
        assert call(**b) == ARG, b


def test_mask_definition():
    """The vectorised mask of the tests against the scalar generator."""
    rows, cols, p, seed, offset = 5, 11, 0.4, 2609, (1 << 64) - 3
    got = keep_mask(rows, cols, p, seed, offset)
    key = W.stream_key(seed, 4)
    assert key == W.mix64((seed + 5 * W.GOLDEN) & W.MASK64)
    for t in range(rows):
        for i in range(cols):
            v = W.raw64(key, (offset + t * 3 + i // 4) & W.MASK64)
            assert got[t, i] == (((v >> (16 * (i % 4))) & 0xFFFF) >= round(p * 65536))
    assert AD.Dropout(0.1, 1, 10).advance(3, 5).offset == 16
