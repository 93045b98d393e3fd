"""The optimizer's entry points on the host (no GPU): exports, refusals, the state's
layout, and what the binding checks before it passes addresses on."""
import ctypes
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_35352_gb300 import build as B
from paper_2609_35352_gb300 import fiona as F
from paper_2609_35352_gb300 import optim as O
from paper_2609_35352_gb300 import workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, PLAN, NODEVICE = F.FIONA_ERR_ARG, F.FIONA_ERR_PLAN, F.FIONA_ERR_NODEVICE


@pytest.fixture(scope="module")
def ctx():
    B.build()
    return F.Context(1024, W.ntt_primes(1024, 40, 1), device=F.FIONA_DEVICE_NONE)


class Tensor(ctypes.Structure):  # fiona_adamw_tensor
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("count", ctypes.c_uint64), ("dtype", ctypes.c_uint32),
                ("group", ctypes.c_uint32)]


class Group(ctypes.Structure):  # fiona_adamw_group
    _fields_ = [(n, ctypes.c_double) for n in ("beta1", "beta2", "eps", "weight_decay", "max_norm")]


def test_exports_and_structures(ctx):
    text = open(os.path.join(ROOT, "include", "fiona_optim.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(fiona_\w+)\s*\(", text)))
    assert names == sorted(O.EXPORTED)
    for n in names:
        assert hasattr(ctypes.CDLL(F.LIB_PATH), n)
    for c, d in ((Tensor, O.TENSOR_DTYPE), (Group, O.GROUP_DTYPE)):
        assert ctypes.sizeof(c) == d.itemsize
        assert all(getattr(c, n).offset == d.fields[n][1] for n, _ in c._fields_)


N, GROUPS = 3, 2
COUNTS, DTYPES = (1000, 0, 300), (2, 1, 0)


class Case:
    """A creation on host memory of the right sizes."""

    def __init__(self, ctx, bits8=False):
        self.ctx, self.flags, self.n_groups, self.n = ctx, 1 if bits8 else 0, GROUPS, N
        self.keep = []
        self.t = (Tensor * N)(*[Tensor(self.room(c * 4), self.room(c * 4), c, d, i % 2) for i, (c, d) in enumerate(zip(COUNTS, DTYPES))])
        self.g = (Group * GROUPS)(*[Group(0.9, 0.999, 1e-8, 0.01, 1.0)] * 2)
        places = 1024 + 512
        self.s = O.State(*[self.room(places * 4) for _ in range(5)], self.room(16), self.room(8), self.room(8))
        if not bits8:
            self.s.m_scale = self.s.v_scale = None

    def room(self, n):
        b = np.zeros(n + 64, np.uint8)
        self.keep.append(b)
        return (b.ctypes.data + 15) // 16 * 16

    def __call__(self, **change):
        h = ctypes.c_void_p()
        a = dict(ctx=self.ctx.handle, n=self.n, t=self.t, n_groups=self.n_groups, g=self.g, flags=self.flags, s=ctypes.byref(self.s), out=ctypes.byref(h))
        a.update(change)
        rc = O.lib().fiona_adamw_create(a["ctx"], a["n"], a["t"], a["n_groups"], a["g"], a["flags"], a["s"], a["out"])
        assert bool(h.value) == (rc == 0)
        if rc == 0:
            self.opt = h
            self.keep.append(h)
        return rc


@pytest.mark.parametrize("bits8", [False, True])
def test_created(ctx, bits8):
    c = Case(ctx, bits8)
    assert c() == 0
    L = O.lib()
    buf = c.room(8 * 2048)
    assert L.fiona_adamw_step(c.opt, None, None) == NODEVICE and L.fiona_adamw_reset(c.opt, None) == NODEVICE
    assert L.fiona_adamw_moments(c.opt, None, 0, buf, None) == NODEVICE and L.fiona_adamw_load_moments(c.opt, None, 0, None, buf) == NODEVICE
    for f in (L.fiona_adamw_moments, L.fiona_adamw_load_moments):
        assert f(c.opt, None, 3, buf, None) == ARG and f(c.opt, None, 0, buf + 8, None) == ARG and f(None, None, 0, buf, None) == ARG
        assert f(c.opt, None, 0, buf, buf + 1024) == ARG and f(c.opt, None, 0, c.s.m, None) == ARG
    assert L.fiona_adamw_step(None, None, None) == ARG and L.fiona_adamw_reset(None, None) == ARG
    L.fiona_adamw_destroy(c.opt)
    L.fiona_adamw_destroy(None)
    # none of these is needed
    for change in (dict(master=None), dict()):
        c = Case(ctx, bits8)
        for k, v in change.items():
            setattr(c.s, k, v)
        assert c() == 0
    c = Case(ctx, bits8)
    c.s.norms = None
    for g in c.g:
        g.max_norm = float("inf")
    assert c() == 0
    assert Case(ctx, bits8)(n=0, t=None) == 0


@pytest.mark.parametrize("bits8", [False, True])
def test_refused(ctx, bits8):
    for k in ("ctx", "t", "g", "s", "out"):
        assert Case(ctx, bits8)(**{k: None}) == ARG, k
    for change in (dict(n_groups=0), dict(n_groups=(1 << 20) + 1), dict(flags=4), dict(n=(1 << 22) + 1)):
        assert Case(ctx, bits8)(**change) == ARG, change
    for k in ("m", "v", "steps", "lr") + (("m_scale", "v_scale") if bits8 else ()):
        c = Case(ctx, bits8)
        setattr(c.s, k, None)
        assert c() == ARG, k
    for k in ("m", "v", "master") + (("m_scale", "v_scale") if bits8 else ()):
        c = Case(ctx, bits8)
        setattr(c.s, k, getattr(c.s, k) + 8)
        assert c() == ARG, k
    for k, off in (("steps", 4), ("lr", 2), ("norms", 2)):
        c = Case(ctx, bits8)
        setattr(c.s, k, getattr(c.s, k) + off)
        assert c() == ARG, k
    if not bits8:
        c = Case(ctx)
        c.s.m_scale = c.room(64)
        assert c() == ARG
    for k, bad in (("beta1", (-0.1, 1.0, float("nan"))), ("beta2", (-0.1, 1.0, float("nan"))), ("eps", (-1.0, 1e-39, float("nan"), float("inf"))),
                   ("weight_decay", (float("nan"), float("inf"))), ("max_norm", (0.0, -1.0, float("nan")))):
        for v in bad:
            c = Case(ctx, bits8)
            setattr(c.g[1], k, v)
            assert c() == ARG, (k, v)
    c = Case(ctx, bits8)
    c.s.norms = None
    assert c() == ARG  # clipped without norms
    c = Case(ctx, bits8)
    c.s.norms = None
    for g in c.g:
        g.max_norm = float("inf")
    c.flags |= 2
    assert c() == ARG
    for k, v in (("param", None), ("grad", None), ("count", (1 << 40) + 1), ("dtype", 3)):
        c = Case(ctx, bits8)
        setattr(c.t[0], k, v)
        assert c() == ARG, k
    for k in ("param", "grad"):
        c = Case(ctx, bits8)
        setattr(c.t[0], k, getattr(c.t[0], k) + 1)
        assert c() == ARG, k
    c = Case(ctx, bits8)
    c.t[2].group = 2
    assert c() == PLAN
    assert F.last_error()


@pytest.mark.parametrize("bits8", [False, True])
def test_overlaps(ctx, bits8):
    """Written ranges against one another and against gradients; gradients may be shared."""
    c = Case(ctx, bits8)
    c.t[2].grad = c.t[0].grad
    assert c() == 0
    for where in ("param", "grad", "m", "v", "master", "steps", "lr", "norms") + (("m_scale", "v_scale") if bits8 else ()):
        for k in ("m", "v", "master", "steps", "norms") + (("m_scale", "v_scale") if bits8 else ()):
            if k == where:
                continue
            c = Case(ctx, bits8)
            setattr(c.s, k, getattr(c.t[0], where) if where in ("param", "grad") else getattr(c.s, where))
            assert c() == PLAN, (k, where)
    for at in (0, 4, 1996):
        c = Case(ctx, bits8)
        c.t[2].param = c.t[0].param + at
        assert c() == PLAN
        c = Case(ctx, bits8)
        c.t[2].grad = c.t[0].param + at
        assert c() == PLAN
    c = Case(ctx, bits8)
    c.t[2].param = c.t[0].param + 2000  # just behind
    assert c() == 0


def test_state_count(ctx):
    n, L = ctypes.c_uint64(), O.lib()
    for counts, want in (((), 0), ((1,), 256), ((256, 0, 257), 768), ((5, 5, 5), 768)):
        t = (Tensor * max(len(counts), 1))(*[Tensor(None, None, c, 0, 0) for c in counts])
        assert L.fiona_adamw_state_count(len(counts), t, ctypes.byref(n)) == 0 and n.value == want
    t = (Tensor * 2)(Tensor(None, None, 1 << 40, 0, 0), Tensor(None, None, 1, 0, 0))
    assert L.fiona_adamw_state_count(2, t, ctypes.byref(n)) == ARG
    assert L.fiona_adamw_state_count(1, None, ctypes.byref(n)) == ARG and L.fiona_adamw_state_count(1, t, None) == ARG


def test_binding(ctx):
    """On a validation-only context the tensors are the host's."""
    def make(**kw):
        a = dict(params=[torch.zeros(4, 100), torch.zeros(7, dtype=torch.bfloat16)], grads=[torch.zeros(4, 100), torch.zeros(7, dtype=torch.bfloat16)])
        a.update(kw)
        return O.AdamW(ctx, a.pop("params"), a.pop("grads"), **a)

    o = make(groups=[[0, 1, 2, 3], 1], lr=[1e-3, 2e-3, 3e-3, 4e-3], max_norm=1.0, state_bits=8, master=True)
    assert o.n_groups == 4 and o.places.tolist() == [0, 256, 512, 768, 1024] and o.m.numel() == 1280 and o.m_scale.numel() == 5
    assert torch.equal(o.lr, torch.tensor([1e-3, 2e-3, 3e-3, 4e-3]))
    with pytest.raises(F.FionaError) as e:
        o.step(active=torch.ones(4, dtype=torch.bool))
    assert e.value.status == NODEVICE
    for bad in (torch.ones(4), torch.ones(3, dtype=torch.bool), torch.ones(8, dtype=torch.bool)[::2]):
        with pytest.raises(ValueError):
            o.step(active=bad)
    for m, v in ((torch.zeros(1279), None), (torch.zeros(1280), torch.zeros(1280).half()), (torch.zeros(2560)[::2], None), (torch.zeros(1280).double(), None)):
        with pytest.raises(ValueError):
            o.moments(m, v)
        with pytest.raises(ValueError):
            o.load_moments(m, v)
    values = torch.zeros(1280)
    for call in (o.moments, o.load_moments):
        for m, v, status in ((values, None, NODEVICE), (o.master, None, ARG), (None, o.master, ARG), (values, values, ARG), (o.norms.new_zeros(0), None, None)):
            with pytest.raises(ValueError if status is None else F.FionaError) as e:
                call(m, v)
            assert status is None or e.value.status == status
    o = make()
    assert o.norms is None and o.master is None and o.n_groups == 1 and o.m.dtype == torch.float32
    assert make(n_groups=5).steps.shape == (5,)
    assert make(params=[], grads=[]).m.numel() == 0
    for bad in (dict(state_bits=16), dict(grads=[torch.zeros(4, 100)]), dict(groups=[0]), dict(groups=[[0, 1, 2], 0]), dict(groups=[-1, 0]),
                dict(groups=[0.5, 0]), dict(groups=[[[0, 1, 2, 3]], 0]), dict(groups=[0, 3], n_groups=2), dict(n_groups=0), dict(n_groups=1.5),
                dict(lr=[1e-3, 1e-3]), dict(lr=[[1e-3]]), dict(grads=[torch.zeros(4, 100), torch.zeros(7)]),
                dict(grads=[torch.zeros(100, 4).t(), torch.zeros(7, dtype=torch.bfloat16)]),
                dict(params=[torch.zeros(100, 4).t(), torch.zeros(7, dtype=torch.bfloat16)]),
                dict(params=[torch.zeros(4, 100, dtype=torch.float64), torch.zeros(7, dtype=torch.bfloat16)],
                     grads=[torch.zeros(4, 100, dtype=torch.float64), torch.zeros(7, dtype=torch.bfloat16)])):
        with pytest.raises(ValueError):
            make(**bad)
    for bad in (dict(betas=(1.0, 0.9)), dict(eps=-1.0), dict(max_norm=0.0), dict(weight_decay=float("nan"))):
        with pytest.raises(F.FionaError):
            make(**bad)
    one = torch.zeros(4, 100)
    with pytest.raises(F.FionaError) as e:  # the same tensor twice
        make(params=[one, one], grads=[torch.zeros(4, 100)] * 2)
    assert e.value.status == PLAN


def test_settings_of_fp32(ctx):
    """An eps and a weight decay that fp32 holds, and none that it would take for infinite."""
    most = float(np.finfo(np.float32).max)
    for k, fine, bad in (("eps", (2.0 ** -126, 1.0, most), (2.0 ** 128, 1e39, 1e300)),
                         ("weight_decay", (most, -most, 1e-300), (2.0 ** 128, -1e39, 1e300))):
        for values, rc in ((fine, F.FIONA_OK), (bad, ARG)):
            for v in values:
                c = Case(ctx, False)
                setattr(c.g[1], k, v)
                assert c() == rc, (k, v)
