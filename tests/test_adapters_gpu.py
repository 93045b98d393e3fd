"""Low-rank adapters beside a shared projection on the GPU, against their
formulas in 64 bits: types, ranks, ragged and empty requests, odd sizes, strides,
dropout, streams, values that are not finite, and the gradients against
differences of the forward pass.

The tolerance of an element is derived (adapter_util.allowed): the rounding of an
fp32 sum over its absolute terms, the two-part operand and the output's type."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

from adapter_util import Reference, check  # noqa: E402

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


def f64(t):
    return None if t is None else t.double().cpu().numpy()


class Problem:
    def __init__(self, ctx, dtype, starts, ids, ranks, r_max, d_in, d_out, seed=0, p=0.0, scales="mixed", base=True,
                 pad=0, scale_x=1.0, scale_dy=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.dtype, dt = ctx, dtype, DT[dtype]
        self.starts, self.ids, self.ranks, self.r_max = starts, ids, ranks, r_max
        self.d_in, self.d_out, self.T, n = d_in, d_out, starts[-1], len(ranks)
        self.scales = [0.5 + 0.75 * (a % 4) - 2.0 * (a % 5 == 4) for a in range(n)] if scales == "mixed" else scales

        def rows(cols, scale=1.0):
            wide = torch.randn(max(self.T, 1), cols + pad, generator=g, device="cuda") * scale
            return wide.to(dt)[:self.T, pad // 2:pad // 2 + cols]

        self.x = rows(d_in, scale_x)
        self.base = rows(d_out, 2.0) if base else None
        self.dy = rows(d_out, scale_dy)
        self.dx_base = rows(d_in, 0.5) if base else None
        self.A = (torch.randn(n, r_max, d_in, generator=g, device="cuda") * d_in ** -0.5).to(dt)
        self.B = (torch.randn(n, d_out, r_max, generator=g, device="cuda") * r_max ** -0.5).to(dt)
        self.drop = AD.Dropout(p, 77 + seed, 1 << 40) if p else None
        self.batch = AD.Batch(ctx, starts, ids, ranks, r_max, self.scales)
        self.work = self.batch.workspace(d_in, d_out, dt)
        self.out = rows(d_out)
        self.dx = rows(d_in)
        self.h = torch.full((self.T, r_max), 7.0, device="cuda")
        self.dA, self.dB = torch.full_like(self.A, 7.0), torch.full_like(self.B, 7.0)

    def reference(self):
        d = None if self.drop is None else (self.drop.p, self.drop.seed, self.drop.offset)
        return Reference(self.starts, self.ids, self.ranks, self.scales, self.r_max, f64(self.x), f64(self.A),
                         f64(self.B), d)

    def forward(self, h=True, stream=None):
        self.batch.forward(self.x, self.A, self.B, self.out, base=self.base, h=self.h if h else None,
                           dropout=self.drop, work=self.work, stream=stream)

    def backward(self, stream=None):
        self.batch.backward(self.x, self.h, self.dy, self.A, self.B, self.dx, self.dA, self.dB,
                            dx_base=self.dx_base, dropout=self.drop, work=self.work, stream=stream)

    def check_forward(self, h=True):
        ref = self.reference()
        value, terms = ref.forward(f64(self.base))
        check("out", self.dtype, f64(self.out), value, terms, self.d_in + self.r_max)
        if h:
            value, terms = ref.hidden()
            check("h", "f32", f64(self.h), value, terms, self.d_in)

    def check_backward(self):
        ref = self.reference()
        dx, dA, dB = ref.backward(f64(self.h), f64(self.dy), f64(self.dx_base))
        check("dx", self.dtype, f64(self.dx), *dx, self.d_out + self.r_max)
        most = max([sum(e - b for b, e, a in zip(self.starts, self.starts[1:], self.ids) if a == j)
                    for j in range(len(self.ranks))], default=0)
        check("dA", self.dtype, f64(self.dA), *dA, self.d_out + most)
        check("dB", self.dtype, f64(self.dB), *dB, most)

    def run_and_check(self):
        self.forward()
        torch.cuda.synchronize()
        self.check_forward()
        self.backward()
        torch.cuda.synchronize()
        self.check_backward()
        assert self.ctx.device_check() == F.FIONA_OK


RAGGED = ([0, 1, 1, 130, 131, 259, 300, 317], [0, 1, 2, 0, -1, 3, 1], [16, 8, 5, 0])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("d_in,d_out", [(256, 384), (64, 8), (1000, 520), (77, 131), (1, 3), (129, 1)])
def test_ragged_requests(ctx, dtype, p, d_in, d_out):
    starts, ids, ranks = RAGGED
    Problem(ctx, dtype, starts, ids, ranks, 16, d_in, d_out, seed=d_in + d_out, p=p).run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("r_max", [1, 3, 8, 24, 33, 64, 72, 128])
def test_ranks(ctx, dtype, r_max):
    ranks = [r_max, max(1, r_max // 2), r_max - 1]
    Problem(ctx, dtype, [0, 140, 290, 301], [1, 0, 2], ranks, r_max, 320, 264, seed=r_max, p=0.1).run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 200])
def test_single_tokens(ctx, dtype, n):
    """One token a request, adapters shared and not, some requests without."""
    rng = np.random.default_rng(n)
    n_ad = max(1, n // 2)
    ids = [int(a) for a in rng.integers(-1, n_ad, n)]
    ranks = [int(r) for r in rng.integers(0, 33, n_ad)]
    pr = Problem(ctx, dtype, list(range(n + 1)), ids, ranks, 32, 768, 1032, seed=n)
    pr.forward(h=False)
    torch.cuda.synchronize()
    pr.check_forward(h=False)
    pr.run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_long_request(ctx, dtype):
    """One adapter over many token tiles, with a short one beside it."""
    Problem(ctx, dtype, [0, 3000, 3001], [1, 0], [16, 16], 16, 512, 640, seed=5, p=0.05).run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [2, 8, 24])
def test_row_strides(ctx, dtype, pad):
    """Column ranges of wider buffers, at whatever alignment their start has."""
    starts, ids, ranks = RAGGED
    Problem(ctx, dtype, starts, ids, ranks, 16, 256, 200, seed=pad, p=0.2, pad=pad).run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_without_base_and_in_place(ctx, dtype):
    starts, ids, ranks = RAGGED
    pr = Problem(ctx, dtype, starts, ids, ranks, 16, 192, 136, base=False, scales=None)
    pr.run_and_check()
    pr = Problem(ctx, dtype, starts, ids, ranks, 16, 192, 136)
    base, dx_base = pr.base.clone(), pr.dx_base.clone()
    pr.out.copy_(base)
    pr.dx.copy_(dx_base)
    pr.base, pr.dx_base = pr.out, pr.dx
    pr.forward()
    pr.backward()
    torch.cuda.synchronize()
    pr.base, pr.dx_base = base, dx_base
    pr.check_forward()
    pr.check_backward()


def test_one_row_for_all(ctx):
    """An input whose rows are one row (stride 0)."""
    pr = Problem(ctx, "bf16", [0, 150], [0], [16], 16, 256, 256)
    pr.x = pr.x[:1].expand(150, 256)
    pr.base = pr.base[:1].expand(150, 256)
    pr.run_and_check()


def test_unused_weights_are_not_read(ctx):
    """Rows of A and columns of B at and above the rank, and adapters without
    rows, may hold anything; gradients are zero there."""
    for dtype in DT:
        pr = Problem(ctx, dtype, [0, 40, 200, 201], [0, 1, 1], [5, 16, 8], 24, 256, 128, p=0.1)
        ref = pr.reference()
        for a, k in enumerate(pr.ranks):
            pr.A[a, k:] = float("nan")
            pr.B[a, :, k:] = float("inf")
        pr.A[2], pr.B[2] = float("nan"), float("nan")
        pr.reference = lambda ref=ref: ref
        pr.run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite_stay_in_their_rows(ctx, dtype):
    """A NaN or an infinity in one request reaches neither another request's rows
    nor another adapter's gradient; a dropped element is zero whatever it held."""
    starts, ids, ranks = [0, 3, 100, 260, 262], [0, 1, -1, 2], [8, 16, 4]
    pr = Problem(ctx, dtype, starts, ids, ranks, 16, 256, 192, p=0.5)
    ref = pr.reference()
    bad = [1, 50, 150]
    pr.x[1, ref.keep[1].argmax()] = float("nan")
    pr.x[50, ref.keep[50].argmin()] = float("inf")  # dropped
    pr.x[150] = float("nan")                         # no adapter: not read
    pr.dy[150] = float("inf")
    pr.dy[261, 7] = float("nan")
    pr.forward()
    pr.backward()
    torch.cuda.synchronize()
    out, dx, dA, dB = f64(pr.out), f64(pr.dx), f64(pr.dA), f64(pr.dB)
    assert np.isnan(out[1]).all() and np.isfinite(np.delete(out, 1, 0)).all()
    assert np.array_equal(out[100:260], f64(pr.base)[100:260])
    assert np.array_equal(dx[100:260], f64(pr.dx_base)[100:260])
    assert np.isfinite(dx[:261]).all() and np.isnan(dx[261][ref.keep[261]]).all()
    assert np.isnan(dA[2, :4][:, ref.keep[261]]).all() and not np.isfinite(dB[0, :, :8]).all()
    assert np.isfinite(dA[1]).all() and np.isfinite(dB[1]).all()
    assert np.isfinite(f64(pr.h)[np.setdiff1d(np.arange(262), [1])]).all() and bad


@pytest.mark.parametrize("scale_x,scale_dy,scale_a", [(2.0 ** 9, 2.0 ** -13, 1.0), (2.0 ** -12, 2.0 ** 8, 1.0),
                                                      (2.0 ** 12, 2.0 ** -4, 2.0 ** 5)])
def test_fp16_range(ctx, scale_x, scale_dy, scale_a):
    """Sums far outside fp16's normal range between the two products."""
    pr = Problem(ctx, "f16", [0, 130, 400], [0, 1], [8, 16], 16, 512, 256, scale_x=scale_x, scale_dy=scale_dy,
                 scales=[2.0 ** -6, 2.0 ** -8], base=False)
    pr.A.mul_(scale_a)
    pr.B.mul_(2.0 ** -5)
    pr.run_and_check()


def test_empty(ctx):
    pr = Problem(ctx, "bf16", [0, 0, 0], [0, 1], [8, 4], 8, 64, 64)
    pr.run_and_check()
    assert not pr.dA.any() and not pr.dB.any()
    pr = Problem(ctx, "bf16", [0, 20], [-1], [], 8, 64, 64)
    pr.run_and_check()
    assert torch.equal(pr.out, pr.base)
    pr = Problem(ctx, "f32", [0], [], [3], 8, 64, 64)
    pr.run_and_check()


def test_same_results_every_time(ctx):
    """No result depends on the order in which blocks run."""
    for dtype in DT:
        pr = Problem(ctx, dtype, [0, 700, 1500, 1600], [0, 1, 0], [16, 13], 16, 520, 264, p=0.1)
        pr.forward()
        pr.backward()
        first = [t.clone() for t in (pr.out, pr.h, pr.dx, pr.dA, pr.dB)]
        for _ in range(5):
            pr.work.fill_(255)
            pr.forward()
            pr.backward()
            for a, b in zip(first, (pr.out, pr.h, pr.dx, pr.dA, pr.dB)):
                assert torch.equal(a, b)


def test_other_streams_and_batches(ctx):
    """Two batches with a workspace each on two streams at once, and a graph."""
    a = Problem(ctx, "bf16", [0, 500], [0], [16], 16, 512, 512, seed=1, p=0.1)
    b = Problem(ctx, "f16", list(range(65)), [i % 9 for i in range(64)], [8] * 9, 8, 512, 512, seed=2)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        a.forward(stream=s1)
        b.forward(stream=s2)
        a.backward(stream=s1)
        b.backward(stream=s2)
    torch.cuda.synchronize()
    for pr in (a, b):
        pr.check_forward()
        pr.check_backward()
        pr.out.zero_()
        pr.dx.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        a.forward(stream=s)
        a.backward(stream=s)
        b.forward(stream=s)
    graph.replay()
    torch.cuda.synchronize()
    a.check_forward()
    a.check_backward()
    b.check_forward()


def test_gradients_are_differences(ctx):
    """The loss sum(out * dy) is linear in each of x, A and B: its difference
    over a step of any length is the gradient's product with the step, up to the
    rounding of the forward pass."""
    pr = Problem(ctx, "f32", [0, 40, 90, 300], [0, 1, 0], [8, 5], 8, 96, 72, p=0.25, base=False)
    pr.forward()
    pr.backward()
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(9)
    for t, grad in ((pr.x, pr.dx), (pr.A, pr.dA), (pr.B, pr.dB)):
        step = torch.randn(t.shape, generator=g, device="cuda")
        keep, loss, size = t.clone(), [], 0.0
        for sign in (1.0, -1.0):
            t.copy_(keep + sign * step)
            pr.forward()
            torch.cuda.synchronize()
            loss.append(float((pr.out.double() * pr.dy.double()).sum()))
            size += float((f64(pr.dy).__abs__() * pr.reference().forward(None)[1]).sum())
        t.copy_(keep)
        want = float((grad.double() * step.double()).sum())
        # the step itself rounds once (keep + step), every sum as in `allowed`
        assert abs((loss[0] - loss[1]) / 2 - want) <= size * 2 * (96 + 72 + 300 + 16) * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("starts,ids", [([0, 700, 900], [0, 1]), (list(range(41)), [i % 2 for i in range(40)])])
def test_order_on_a_stream(ctx, dtype, starts, ids):
    """A call follows what was queued before it, and what is queued after follows
    the call: inputs that a slow kernel writes just before, and overwrites just after."""
    pr = Problem(ctx, dtype, starts, ids, [16, 8], 16, 1024, 768, seed=3, p=0.1)
    pr.forward()
    pr.backward()
    torch.cuda.synchronize()
    first = [t.clone() for t in (pr.out, pr.h, pr.dx, pr.dA, pr.dB)]
    inputs = [pr.x, pr.base, pr.dy, pr.dx_base, pr.A, pr.B]
    good = [t.clone() for t in inputs]
    slow = torch.randn(4096, 4096, device="cuda")
    for _ in range(3):
        for t in inputs + [pr.out, pr.h, pr.dx, pr.dA, pr.dB]:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        torch.mm(slow, slow)
        for t, g in zip(inputs, good):
            t.copy_(g)
        pr.forward()
        pr.backward()
        for t in inputs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        for a, b in zip(first, (pr.out, pr.h, pr.dx, pr.dA, pr.dB)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d_in,d_out,r_max,pad", [(1001, 777, 43, 0), (1024, 777, 24, 0), (1001, 768, 33, 5), (640, 512, 100, 3)])
def test_odd_sizes_of_long_batches(ctx, dtype, d_in, d_out, r_max, pad):
    """Widths, ranks and strides that are no multiples of eight, with enough rows
    that copies for the tensor cores pay."""
    pr = Problem(ctx, dtype, [0, 1800, 1803, 1900, 4000], [0, 1, -1, 2], [r_max, r_max - 2, 7], r_max, d_in, d_out,
                 seed=r_max, p=0.1, pad=pad)
    pr.run_and_check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("starts,ids", [([0, 299, 300], [0, 1]), (list(range(41)), [i % 3 - 1 for i in range(40)])])
@pytest.mark.parametrize("d_in,d_out,shift", [(256, 136, 8), (77, 131, 3)])
def test_rows_past_32_bits(ctx, dtype, starts, ids, d_in, d_out, shift):
    """Rows so far apart that the last lie more than 2^32 elements on, all of them
    columns of one buffer."""
    T = starts[-1]
    ld = (5 << 30) // T // 64 * 64 + shift
    assert (T - 1) * ld > 1 << 32
    pr = Problem(ctx, dtype, starts, ids, [16, 9], 16, d_in, d_out, seed=T, p=0.2)
    wide, at = torch.empty(T * ld, dtype=DT[dtype], device="cuda").view(T, ld), 0
    for name in ("x", "base", "dy", "dx_base", "out", "dx"):
        t = getattr(pr, name)
        view = wide[:, at:at + t.shape[1]]
        view.copy_(t)
        setattr(pr, name, view)
        at += (t.shape[1] + 7) // 8 * 8 + shift
    pr.run_and_check()


@pytest.mark.parametrize("dtype,starts", [("bf16", [0, 300]), ("f16", [0, 130]), ("bf16", list(range(9))), ("f32", list(range(9)))])
def test_waits_that_run_out_are_reported(ctx, dtype, starts, monkeypatch):
    """Kernels whose barriers expect an arrival that never comes give up, end and
    say so; the context goes on."""
    ids = [0] * (len(starts) - 1)
    monkeypatch.setenv("FIONA_ADAPTER_TEST_STALL", "1")
    stalled = Problem(ctx, dtype, starts, ids, [32], 32, 512, 384, p=0.1)
    monkeypatch.delenv("FIONA_ADAPTER_TEST_STALL")
    for call in (stalled.forward,) if len(starts) > 2 else (stalled.forward, stalled.backward):
        assert ctx.device_check() == F.FIONA_OK
        call()
        assert ctx.device_check() == F.FIONA_ERR_TIMEOUT
    Problem(ctx, dtype, starts, ids, [32], 32, 512, 384, p=0.1).run_and_check()
