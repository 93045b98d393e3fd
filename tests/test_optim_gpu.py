"""AdamW over many tensors against the formulas in 64 bits (optim_util.py derives what
rounding may do)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import optim as O  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

import optim_util as OU  # noqa: E402

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAME = {v: k for k, v in DT.items()}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


def f64(t):
    return t.double().cpu().numpy()


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def tensors(shapes, dtypes, seed, offset=0):
    """Weights and gradients, `offset` elements behind an allocation's start."""
    params, grads = [], []
    for i, (shape, dt) in enumerate(zip(shapes, dtypes)):
        n = int(np.prod(shape))
        for out, scale in ((params, 0.05), (grads, 0.01 * (1 + i))):
            flat = torch.zeros(n + offset, dtype=dt, device="cuda")
            t = flat[offset:].view(shape)
            t.copy_(normal(shape, dt, seed + 2 * i + (out is grads), scale))
            out.append(t)
    return params, grads


class Model:
    """An optimizer beside its formulas: tensors' slices as segments."""

    def __init__(self, ctx, params, grads, groups, settings, **kw):
        self.params, self.grads, self.settings = params, grads, settings
        n = len(settings)
        clip = any(np.isfinite(s.max_norm) for s in settings) or kw.pop("norms", False)
        self.opt = O.AdamW(ctx, params, grads, groups=groups, lr=[s.lr for s in settings],
                           betas=([s.beta1 for s in settings], [s.beta2 for s in settings]), eps=[s.eps for s in settings],
                           weight_decay=[s.weight_decay for s in settings], max_norm=[s.max_norm for s in settings] if clip else None,
                           n_groups=n, **kw)
        self.segments = []  # (tensor, slice or None, group)
        for i, p in enumerate(params):
            of = 0 if groups is None else groups[i]
            if np.ndim(of):
                self.segments += [(i, k, g) for k, g in enumerate(of)]
            else:
                self.segments.append((i, None, of))
        self.counts = [p.numel() if k is None else p[k].numel() for p, k in ((params[i], k) for i, k, _ in self.segments)]
        self.places, self.total = OU.places(self.counts)
        assert (self.opt.places == self.places).all() and self.opt.m.numel() == self.total
        self.bits8 = self.opt.m.dtype == torch.int8

    def start(self, seed, steps):
        """Moments and step counts of a training under way."""
        o = self.opt
        inside = torch.zeros(self.total, device="cuda")
        for at, n in zip(self.places, self.counts):
            inside[at:at + n] = 1.0
        m = normal((self.total,), torch.float32, seed, 3e-3) * inside
        v = (normal((self.total,), torch.float32, seed + 1, 1e-2) * inside).square()
        o.load_moments(m, v, stream=torch.cuda.current_stream())
        o.steps.copy_(torch.tensor(steps))
        if o.master is not None:
            o.master.mul_(1 + 1e-4 * normal((self.total,), torch.float32, seed + 2))

    def snapshot(self):
        o = self.opt
        s = {"m": o.m, "v": o.v, "steps": o.steps, "master": o.master, "m_scale": o.m_scale, "v_scale": o.v_scale}
        return dict({k: None if t is None else t.cpu().numpy().copy() for k, t in s.items()}, params=[f64(p) for p in self.params])

    def values(self, s):
        if not self.bits8:
            return s["m"].astype(np.float64), s["v"].astype(np.float64)
        rep = np.repeat(np.arange(self.total // OU.BLOCK), OU.BLOCK)
        return OU.decode_m(s["m"], s["m_scale"].astype(np.float64)[rep]), OU.decode_v(s["v"], s["v_scale"].astype(np.float64)[rep])

    def check_step(self, active=None):
        before = self.snapshot()
        grads = [f64(g) for g in self.grads]
        self.opt.step(active=None if active is None else torch.tensor(active, device="cuda"), stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        after = self.snapshot()
        m0, v0 = self.values(before)
        live = [active is None or active[g] for g in range(len(self.settings))]
        mine = [[grads[i] if k is None else grads[i][k] for i, k, h in self.segments if h == g] for g in range(len(self.settings))]
        norms = [OU.norm_of(x) if on else 0.0 for x, on in zip(mine, live)]
        if self.opt.norms is not None:
            OU.check("norms", "f32", f64(self.opt.norms), np.array(norms), 60 * OU.U * np.array(norms))
        assert (after["steps"] == before["steps"] + np.array(live, dtype=np.int64)).all()
        want_m, want_v = np.zeros(self.total), np.zeros(self.total)
        dm, dv = np.zeros(self.total), np.zeros(self.total)
        untouched = np.ones(self.total, bool)
        for (i, k, g), at, n in zip(self.segments, self.places, self.counts):
            where = slice(at, at + n)
            dt = NAME[self.params[i].dtype]
            old, new = ((x["params"][i] if k is None else x["params"][i][k]).reshape(-1) for x in (before, after))
            if not live[g]:
                assert np.array_equal(old, new)
                continue
            untouched[where] = False
            master = self.opt.master is not None and dt != "f32"
            w = before["master"][where].astype(np.float64) if master else old
            grad = (grads[i] if k is None else grads[i][k]).reshape(-1)
            (w1, dw), (m1, dm1), (v1, dv1) = OU.step(self.settings[g], int(after["steps"][g]), w, m0[where], v0[where], grad,
                                                     norms[g] if self.opt.norms is not None else None)
            if master:
                OU.check("master", "f32", after["master"][where], w1, dw)
                # the weights are the masters, rounded
                assert np.array_equal(new, f64(torch.from_numpy(after["master"][where]).to(self.params[i].dtype)))
            else:
                OU.check("weights %d" % i, dt, new, w1, dw)
            want_m[where], want_v[where], dm[where], dv[where] = m1, v1, dm1, dv1
        if self.bits8:
            b = OU.BLOCK
            rows = ~untouched.reshape(-1, b).all(1)
            u = np.sqrt(want_v)
            du = np.minimum(dv / np.maximum(u, 1e-300), np.sqrt(2 * dv)) + 4 * OU.U * u
            pick = lambda x: x.reshape(-1, b)[rows]  # noqa: E731
            OU.check_codes("m", pick(after["m"]), after["m_scale"][rows], pick(want_m), pick(dm), 127)
            OU.check_codes("v", pick(after["v"]), after["v_scale"][rows], pick(u), pick(du), 255)
            for k in ("m_scale", "v_scale"):
                assert np.array_equal(after[k][~rows], before[k][~rows])
        else:
            OU.check("m", "f32", after["m"][~untouched], want_m[~untouched], dm[~untouched])
            OU.check("v", "f32", after["v"][~untouched], want_v[~untouched], dv[~untouched])
        for k in ("m", "v") + (("master",) if self.opt.master is not None else ()):
            assert np.array_equal(after[k][untouched], before[k][untouched]), k
        return norms


SHAPES = [(1,), (3, 5), (7, 64), (256,), (1024,), (1025,), (3, 333, 7), (2048, 3), (4099,), (0, 4), (16, 96, 8), (700, 33)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "mixed"])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_one_model(ctx, bits, master, dtype, offset):
    dtypes = [DT[dtype]] * len(SHAPES) if dtype != "mixed" else [list(DT.values())[i % 3] for i in range(len(SHAPES))]
    params, grads = tensors(SHAPES, dtypes, 1, offset)
    m = Model(ctx, params, grads, None, [OU.Group(1e-3)], state_bits=bits, master=master)
    m.check_step()  # (from zero)
    m.check_step()
    m.start(50, [1234])
    m.check_step()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_many_models(ctx, bits, master):
    """Clients' slices of shared tensors beside whole tensors: settings, norms, step counts
    and clipping by group, groups that sit out, one without tensors."""
    clients = 5
    shapes = [(clients, 8, 96), (clients, 33, 8), (clients, 13, 77), (700,), (clients, 1024)]
    params, grads = tensors(shapes, [torch.bfloat16, torch.bfloat16, torch.float16, torch.float32, torch.float32], 3)
    groups = [list(range(clients)), [4, 3, 2, 1, 0], list(range(clients)), 2, [1, 1, 0, 5, 5]]
    settings = [OU.Group(1e-3), OU.Group(5e-4, 0.8, 0.99, 1e-6, 0.1, 0.5), OU.Group(2e-3, max_norm=0.1), OU.Group(0.0, 0.0, 0.0, 1e-3, 0.0, 1e9),
                OU.Group(1e-2, weight_decay=-0.1), OU.Group(1e-3, max_norm=1e-3), OU.Group(1e-3)]
    m = Model(ctx, params, grads, groups, settings, state_bits=bits, master=master)
    m.start(70, [1, 5, 100, 100000, 3000, 10 ** 7, 0])
    norms = m.check_step()
    assert norms[1] > 0.5 and norms[2] > 0.1 and norms[3] < 1e9 and norms[6] == 0
    m.check_step(active=[True, False, True, False, True, False, False])
    m.check_step(active=[False] * 7)
    m.check_step()


@pytest.mark.parametrize("bits", [32, 8])
def test_sizes_at_random(ctx, bits):
    rng = np.random.default_rng(2609 + bits)
    for i in range(12):
        n, clients = int(rng.integers(1, 6)), int(rng.integers(1, 9))
        shapes = [(clients,) + tuple(int(x) for x in np.exp(rng.uniform(0, 4.5, int(rng.integers(1, 3))))) for _ in range(n)]
        dtypes = [list(DT.values())[int(rng.integers(0, 3))] for _ in range(n)]
        params, grads = tensors(shapes, dtypes, 100 * i, int(rng.integers(0, 9)))
        settings = [OU.Group(1e-3, max_norm=float(np.exp(rng.uniform(-5, 3)))) for _ in range(clients)]
        m = Model(ctx, params, grads, [list(range(clients))] * n, settings, state_bits=bits, master=bool(rng.random() < 0.5))
        m.start(i, [int(x) for x in rng.integers(0, 1000, clients)])
        m.check_step()
        m.check_step(active=[bool(x) for x in rng.random(clients) < 0.7])


def state_of(o, params):
    return [t.clone() for t in list(params) + [o.m, o.v, o.steps] + [x for x in (o.master, o.m_scale, o.v_scale, o.norms) if x is not None]]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_do_not_depend_on_their_company(ctx, bits):
    """A tensor steps the same alone as among others (bit for bit), wherever it stands."""
    shapes = [(33, 7), (4096,), (5000,), (64, 64)]
    params, grads = tensors(shapes, [torch.bfloat16] * 4, 5)
    alone = [p.clone() for p in params]
    shifted = []
    for p in params:
        flat = torch.zeros(p.numel() + 1, dtype=p.dtype, device="cuda")
        flat[1:].copy_(p.view(-1))
        shifted.append(flat[1:])
    for step in range(3):
        if step == 0:
            together = O.AdamW(ctx, params, grads, state_bits=bits)
            each = [O.AdamW(ctx, [p], [g], state_bits=bits) for p, g in zip(alone, grads)]
            moved = O.AdamW(ctx, shifted, [g.reshape(-1) for g in grads], state_bits=bits)
        s = torch.cuda.current_stream()
        together.step(stream=s)
        moved.step(stream=s)
        for o in each:
            o.step(stream=s)
        assert same(params, alone) and all(torch.equal(p.view(-1), q) for p, q in zip(params, shifted))
        assert torch.equal(together.m, moved.m) and torch.equal(together.v, moved.v)


class Stepwise:
    """Moments in 8 bits by the formulas step by step in fp32 (numpy: each operation rounded
    to nearest by itself), blocks [n][256]."""
    f = np.float32

    @classmethod
    def decode(cls, m8, v8, ms, vs):
        q, r = m8.astype(cls.f), v8.astype(cls.f)
        u = (r * r) * (vs * (cls.f(1) / cls.f(65025)))
        return (q * np.abs(q)) * (ms * (cls.f(1) / cls.f(16129))), u * u

    @classmethod
    def encode(cls, value, top):
        scale = np.abs(value).max(1, keepdims=True)
        y = (np.abs(value) / np.maximum(scale, cls.f(1e-30))) * cls.f(top * top) - cls.f(0.25)
        q = np.rint(np.sqrt(np.maximum(y, cls.f(0))))
        q = np.where(value > 0, np.maximum(q, 1), 0) if top == 255 else np.copysign(q, value)
        return q.astype(np.int8 if top == 127 else np.uint8), scale

    @classmethod
    def step(cls, m8, v8, ms, vs, g, beta1, beta2):
        m, v = cls.decode(m8, v8, ms, vs)
        m = cls.f(beta1) * m + cls.f(1 - beta1) * g
        v = cls.f(beta2) * v + cls.f(1 - beta2) * (g * g)
        return cls.encode(m, 127) + cls.encode(np.sqrt(v), 255)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [None, 0.5])
@pytest.mark.parametrize("rows", [200, 9000])
def test_codes_step_by_step(ctx, dtype, max_norm, rows):
    """Every code and scale of three steps is that of the formulas evaluated operation by
    operation, none a border further (a clipped gradient's factor goes by a norm that is as
    good as from fp64)."""
    n = rows * 256
    p, g = normal((n,), DT[dtype], 1, 0.02), normal((n,), DT[dtype], 2, 1e-3)
    o = O.AdamW(ctx, [p], [g], state_bits=8, max_norm=max_norm)
    s = torch.cuda.current_stream()
    o.load_moments(normal((n,), torch.float32, 3, 3e-4), (normal((n,), torch.float32, 4, 1e-3)).square(), stream=s)
    state = [t.cpu().numpy() for t in (o.m.view(-1, 256), o.v.view(-1, 256), o.m_scale.view(-1, 1), o.v_scale.view(-1, 1))]
    for k in range(3):
        grad = g.float().cpu().numpy().reshape(-1, 256)
        if max_norm is not None:
            norm = np.sqrt((grad.astype(np.float64) ** 2).sum())
            grad = grad * np.float32(min(1.0, max_norm / norm))
            assert (norm > max_norm) == (rows == 9000)
        m8, ms, v8, vs = Stepwise.step(*state, grad, 0.9, 0.999)
        o.step(stream=s)
        torch.cuda.synchronize()
        got = [t.cpu().numpy() for t in (o.m.view(-1, 256), o.v.view(-1, 256), o.m_scale.view(-1, 1), o.v_scale.view(-1, 1))]
        assert np.array_equal(got[2], ms) and np.array_equal(got[3], vs)
        assert np.array_equal(got[0], m8) and np.array_equal(got[1], v8)
        state = got
        g.copy_(normal((n,), DT[dtype], 10 + k, 1e-3))
    # what is loaded is rounded the same way, and read out as it stands
    values = [torch.empty(n, device="cuda") for _ in range(2)]
    o.moments(*values, stream=s)
    torch.cuda.synchronize()
    want = Stepwise.decode(*got)
    assert np.array_equal(values[0].cpu().numpy(), want[0].reshape(-1)) and np.array_equal(values[1].cpu().numpy(), want[1].reshape(-1))
    fresh = normal((n,), torch.float32, 20), normal((n,), torch.float32, 21).square()
    o.load_moments(*fresh, stream=s)
    for x, codes, scale, top in ((fresh[0], o.m, o.m_scale, 127), (fresh[1].sqrt(), o.v, o.v_scale, 255)):
        q, want = Stepwise.encode(x.cpu().numpy().reshape(-1, 256), top)
        assert np.array_equal(scale.cpu().numpy(), want.reshape(-1)) and np.array_equal(codes.cpu().numpy().reshape(-1, 256), q)


@pytest.mark.parametrize("bits", [32, 8])
def test_not_finite(ctx, bits):
    """A gradient that is not finite: with skip_nonfinite its group sits the step out; without,
    what the formula gives, in its own group."""
    for bad in (float("inf"), float("nan"), float("-inf")):
        shapes = [(3, 700)]
        params, grads = tensors(shapes, [torch.bfloat16], 8)
        m = Model(ctx, params, grads, [[0, 1, 2]], [OU.Group(1e-3, max_norm=1.0)] * 3, state_bits=bits, skip_nonfinite=True)
        m.start(3, [5, 6, 7])
        before = state_of(m.opt, params)
        keep = grads[0].clone()
        grads[0][1, 300] = bad
        m.opt.step(stream=torch.cuda.current_stream())
        assert m.opt.steps.tolist() == [6, 6, 8]
        norms = m.opt.norms.tolist()
        assert not np.isfinite(norms[1]) and np.isfinite([norms[0], norms[2]]).all()
        assert torch.equal(params[0][1], before[0][1]) and not torch.equal(params[0][0], before[0][0])
        at, n = m.places[1], 768
        assert torch.equal(m.opt.m[at:at + n], before[1][at:at + n]) and torch.equal(m.opt.v[at:at + n], before[2][at:at + n])
        # without: NaN where the formula has it, other groups as they would be
        clean = [p.clone() for p in params]
        for skip, p, g in ((False, params, grads), (False, clean, [keep])):
            o = O.AdamW(ctx, p, g, groups=[[0, 1, 2]], state_bits=bits, skip_nonfinite=skip)
            o.step(stream=torch.cuda.current_stream())
        assert torch.equal(params[0][0], clean[0][0]) and torch.equal(params[0][2], clean[0][2])
        assert torch.isnan(params[0][1, 300])
        if bits == 32:  # (in 8 bits a block shares a scale)
            assert torch.equal(params[0][1, :300], clean[0][1, :300])
        else:
            mm, vv = torch.empty(o.m.numel(), device="cuda"), torch.empty(o.m.numel(), device="cuda")
            o2 = O.AdamW(ctx, params, grads, groups=[[0, 1, 2]], state_bits=8)
            o2.step(stream=torch.cuda.current_stream())
            o2.moments(mm, vv, stream=torch.cuda.current_stream())
            assert torch.isnan(mm[768 + 256:768 + 512]).all() and torch.isfinite(mm[:768]).all()


def test_norms_without_clipping(ctx):
    """max_norm infinity: norms are taken, nothing is clipped; gradients of 0; a norm past
    fp32's squares counts as infinite."""
    params, grads = tensors([(5000,), (3,)], [torch.float32] * 2, 1)
    m = Model(ctx, params, grads, None, [OU.Group()], norms=True)
    m.check_step()
    for g in grads:
        g.zero_()
    m.check_step()
    grads[0][7] = 1e25
    o = O.AdamW(ctx, params, grads, max_norm=1.0, skip_nonfinite=True)
    before = params[0].clone()
    o.step(stream=torch.cuda.current_stream())
    assert o.norms.tolist() == [float("inf")] and o.steps.tolist() == [0] and torch.equal(before, params[0])


def test_extreme_moments(ctx):
    """8 bits: blocks of zeros, of one value, of values far apart, and very small ones; a
    second moment above zero never falls to code 0."""
    n = 256 * 8
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    o = O.AdamW(ctx, [p], [g], state_bits=8)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m[256:512], v[256:512] = 0.5, 0.25
    m[512:768] = torch.logspace(-30, 0, 256, device="cuda") * torch.tensor([1.0, -1.0], device="cuda").repeat(128)
    v[512:768] = torch.logspace(-30, 0, 256, device="cuda")
    m[768:1024], v[768:1024] = 1e-31, 2e-38  # (m below 2^-100; v normal)
    m[1024:1280], v[1024:1280] = 3e38, 3e38
    v[1280:1536] = 1e-42  # below 2^-126
    s = torch.cuda.current_stream()
    o.load_moments(m, v, stream=s)
    gm, gv = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    o.moments(gm, gv, stream=s)
    u = f64(v).copy()
    u[1280:1536] = 0.0
    want_m = f64(m).copy()
    want_m[768:1024] = 0.0
    OU.check_codes("m", o.m.cpu().numpy(), o.m_scale.cpu().numpy(), want_m, 4 * OU.U * np.abs(want_m), 127)
    OU.check_codes("v", o.v.cpu().numpy(), o.v_scale.cpu().numpy(), np.sqrt(u), 4 * OU.U * np.sqrt(u), 255)
    assert (gm[:256] == 0).all() and (gv[:256] == 0).all() and (gv[512:768] > 0).all() and (gv[1280:1536] == 0).all()
    assert (gm[256:512] - 0.5).abs().max() < 1e-6 and (gv[256:512] - 0.25).abs().max() < 1e-6
    # what a code stands for is found again
    codes = [o.m.clone(), o.v.clone()]
    o.load_moments(gm, gv, stream=s)
    assert torch.equal(o.m, codes[0]) and torch.equal(o.v, codes[1])
    scales = [o.m_scale.clone(), o.v_scale.clone()]
    half = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    o.moments(half[0], None, stream=s)
    o.moments(None, half[1], stream=s)
    assert torch.equal(half[0], gm.bfloat16()) and torch.equal(half[1], gv.bfloat16())
    # a block with a NaN
    m[300] = float("nan")
    o.load_moments(m, None, stream=s)
    o.moments(gm, gv, stream=s)
    assert torch.isnan(gm[256:512]).all() and torch.isfinite(gm[:256]).all() and torch.isfinite(gm[512:]).all()
    assert torch.equal(o.v_scale, scales[1])


def test_reset_and_checkpoints(ctx):
    """A state saved and put back goes on as if nothing had been; reset starts over."""
    for bits in (32, 8):
        params, grads = tensors([(3, 1000), (77,)], [torch.bfloat16] * 2, 4)
        first = [p.clone() for p in params]
        o = O.AdamW(ctx, params, grads, state_bits=bits, master=True, max_norm=0.5)
        s = torch.cuda.current_stream()
        for _ in range(3):
            o.step(stream=s)
        saved = {k: getattr(o, k).clone() for k in ("m", "v", "m_scale", "v_scale", "master", "steps") if getattr(o, k) is not None}
        kept = [p.clone() for p in params]
        for _ in range(2):
            o.step(stream=s)
        want = state_of(o, params)
        for k, t in saved.items():
            getattr(o, k).copy_(t)
        for p, t in zip(params, kept):
            p.copy_(t)
        for _ in range(2):
            o.step(stream=s)
        assert same(want, state_of(o, params))
        for p, t in zip(params, first):
            p.copy_(t)
        o.reset(stream=s)
        assert o.steps.tolist() == [0] and (o.m == 0).all() and (o.v == 0).all()
        assert torch.equal(o.master[:3000], first[0].view(-1).float()) and (o.master[3000:int(o.places[1])] == 0).all()
        for _ in range(5):
            o.step(stream=s)
        assert same(want, state_of(o, params))


@pytest.mark.parametrize("bits", [32, 8])
def test_streams_and_graphs(ctx, bits):
    """A captured step replayed, with learning rate, activity and gradients changed in
    between, is the eager steps; on another stream too."""
    def make():
        params, grads = tensors([(4, 16, 96), (4, 33)], [torch.bfloat16, torch.float32], 6)
        o = O.AdamW(ctx, params, grads, groups=[[0, 1, 2, 3], [0, 1, 2, 3]], max_norm=0.2, state_bits=bits, master=True)
        return params, grads, o, torch.ones(4, dtype=torch.uint8, device="cuda")

    def change(k, grads, o, active):
        o.lr.fill_(1e-3 / (k + 1))
        active.copy_(torch.tensor([1, k % 2, 1, 0 if k == 2 else 1], dtype=torch.uint8))
        grads[0].mul_(-0.5)

    runs = []
    for how in ("eager", "stream", "graph"):
        params, grads, o, active = make()
        torch.cuda.synchronize()
        if how == "graph":
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                o.step(active=active, stream=torch.cuda.current_stream())
        side = torch.cuda.Stream()
        for k in range(4):
            if how == "stream":
                with torch.cuda.stream(side):
                    change(k, grads, o, active)
                    o.step(active=active, stream=side)
            else:
                change(k, grads, o, active)
                graph.replay() if how == "graph" else o.step(active=active, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        runs.append(state_of(o, params))
    assert same(runs[0], runs[1]) and same(runs[0], runs[2])
    assert runs[0][4].tolist() == [4, 2, 4, 3]


def test_many_elements(ctx):
    """Places past 32 bits: the last of 4.4e9 elements step as they would alone."""
    n = (1 << 32) + 70000
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-5000:], g[-5000:] = normal((5000,), torch.bfloat16, 1), normal((5000,), torch.bfloat16, 2)
    o = O.AdamW(ctx, [p], [g], state_bits=8, max_norm=1.0)
    q, h = p[-5000 - (n - 5000) % 256:].clone(), g[-5000 - (n - 5000) % 256:].clone()
    alone = O.AdamW(ctx, [q], [h], state_bits=8, max_norm=1.0)
    s = torch.cuda.current_stream()
    for _ in range(2):
        o.step(stream=s)
        alone.step(stream=s)
    assert abs(float(o.norms) / float(alone.norms) - 1) < 1e-6
    # (the two sums of squares may be cut into pieces differently)
    assert (p[-5000:].float() - q[-5000:].float()).abs().max() <= 2.0 ** -7 * q.float().abs().max()
    k = q.numel()
    tail = o.m[(n + 255) // 256 * 256 - (k + 255) // 256 * 256:][:k]
    assert (tail.int() - alone.m[:k].int()).abs().max() <= 1
    assert (o.m[:1 << 20] == 0).all() and (p[:1 << 20] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits,master", [(32, False), (8, False), (8, True)])
@pytest.mark.parametrize("n", [300, 5000, 6_000_000])
def test_squares_past_fp32(ctx, dtype, bits, master, n):
    """A finite gradient whose square is infinite: v is, so the step is none and decay alone moves
    its weight, in either width of the moments; other weights are as without it."""
    p, g = normal((n,), DT[dtype], 1), normal((n,), DT[dtype], 2, 1e-2)
    q, h = p.clone(), g.clone()
    at = [0, 17, 256 + 3, n - 1]
    for i in at[:-1]:
        g[i] = 2e19
    g[at[-1]] = -3e38
    s = torch.cuda.current_stream()
    opts = [O.AdamW(ctx, [w], [d], lr=0.1, state_bits=bits, master=master) for w, d in ((p, g), (q, h))]
    old = p.clone()
    for o in opts:
        o.step(stream=s)
    w = f64(old)[at]
    # (lr and weight decay are rounded, then their product and the weight)
    OU.check("weights", dtype, f64(p)[at], w - 0.1 * 0.01 * w, 4 * OU.U * 0.001 * np.abs(w) + OU.U * np.abs(w))
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[at] = False
    assert torch.equal(p[keep], q[keep])
    if bits == 8:
        blocks = sorted({i // 256 for i in at})
        for o in opts[:1]:
            scales = torch.stack([o.m_scale, o.v_scale])
            assert torch.isnan(scales[:, blocks]).all()
            others = [b for b in range(scales.shape[1]) if b not in blocks]
            assert torch.equal(scales[:, others], torch.stack([opts[1].m_scale, opts[1].v_scale])[:, others])
    else:
        assert torch.isinf(opts[0].v[at]).all() and torch.isfinite(opts[0].m).all()


@pytest.mark.parametrize("groups,offset", [(300, 0), (300, 1), (1600, 0), (1600, 1)])
def test_norms_of_equal_gradients(ctx, groups, offset):
    """4096 equal fp32 gradients c a group, whose squares lose the same in every product: the norm is
    64 c to the last bit, and the factor of clipping the nearest to max_norm / (64 c).  (What the sums
    in two parts leave is some 2^-40 of the norm: of 1900 factors none lies that near a border.)"""
    flat = torch.zeros(groups * 4096 + offset, device="cuda")
    g = flat[offset:].view(groups, 4096)
    c = normal((groups, 1), torch.float32, 7).abs() + 0.01
    g.copy_(c.expand(groups, 4096))
    p = torch.zeros(groups * 4096 + offset, device="cuda")[offset:].view(groups, 4096)
    o = O.AdamW(ctx, [p], [g], groups=[list(range(groups))], betas=(0.0, 0.999), max_norm=0.1)
    o.step(stream=torch.cuda.current_stream())
    c = c[:, 0].cpu().numpy()
    assert np.array_equal(o.norms.cpu().numpy(), c * np.float32(64))
    k = np.minimum(0.1 / (64 * c.astype(np.float64)), 1.0).astype(np.float32)
    assert np.array_equal(o.m.view(groups, 4096).cpu().numpy(), np.broadcast_to((k * c)[:, None], (groups, 4096)))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_norms_to_the_last_bit(ctx, dtype):
    """Norms of gradients of all sizes, some far larger than others, are those of 64 bits, rounded."""
    sizes = [1, 2, 33, 256, 1000, 4096, 70001, 1 << 20] * 20
    grads = [(normal((n,), torch.float32, 40 + i) * torch.exp(normal((n,), torch.float32, 400 + i, 4.0))).clamp(-6e4, 6e4).to(DT[dtype])
             for i, n in enumerate(sizes)]
    params = [torch.zeros_like(g) for g in grads]
    o = O.AdamW(ctx, params, grads, groups=list(range(len(sizes))), max_norm=1.0)
    o.step(stream=torch.cuda.current_stream())
    # (squares are exact in 64 bits, and math.fsum has no error of its own)
    want = [math.sqrt(math.fsum((f64(g) ** 2).tolist())) for g in grads]
    assert np.array_equal(o.norms.cpu().numpy(), np.array(want, dtype=np.float32))


@pytest.mark.parametrize("bits", [32, 8])
def test_last_of_many_elements(ctx, bits):
    """Places past 32 bits, bit for bit: the last of 4.4e9 weights move as they would alone."""
    n, k = (1 << 32) + 70000, 5000
    if torch.cuda.mem_get_info()[0] < (90 << 30):
        pytest.skip("90 GB of device memory")
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    first = (n - k) // 256 * 256
    p[first:], g[first:] = normal((n - first,), torch.bfloat16, 1), normal((n - first,), torch.bfloat16, 2)
    q, h = p[first:].clone(), g[first:].clone()
    old = q.clone()
    s = torch.cuda.current_stream()
    o, alone = (O.AdamW(ctx, [w], [d], lr=0.1, state_bits=bits) for w, d in ((p, g), (q, h)))
    for _ in range(2):
        o.step(stream=s)
        alone.step(stream=s)
    assert float((q != old).float().mean()) > 0.99
    assert torch.equal(p[first:], q)
    for name in ("m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
        end = getattr(alone, name)
        assert torch.equal(getattr(o, name)[-end.numel():], end) and (end != 0).any(), name
    assert (p[:1 << 20] == 0).all() and (o.m[:1 << 20] == 0).all()
