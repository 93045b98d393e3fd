"""Sums of very many terms of one sign.  The accumulator of the tensor cores cuts
every addition toward zero, so a chain of additions loses a part of a sum that grows
evenly, the more the longer it is.  The kernels bound their chains, so that what is lost
does not grow with the batch or the width: h is held to 2^-16 of itself (256 additions
that lose half a unit of 2^-23), 16-bit results to that and the mean of their roundings."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
CHAIN = 2.0 ** -16


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


def mean_off(got, want):
    return abs(float(((got.double() - want) / want).mean()))


def rounding_mean(unit, n):
    """Six deviations of the mean of n roundings, each within `unit` of its value."""
    return 6 * unit / math.sqrt(3 * n)


@pytest.mark.parametrize("dtype,tokens,d,rank", [("f16", 1 << 24, 64, 8), ("bf16", 1 << 22, 64, 16), ("f16", 1 << 22, 128, 72)])
def test_gradients_of_a_very_long_batch(ctx, dtype, tokens, d, rank):
    g, dt = torch.Generator(device="cuda").manual_seed(tokens + rank), DT[dtype]

    def spread(n):  # (so that results, and with them their roundings, spread over an octave)
        return torch.rand(n, generator=g, device="cuda") + 1

    x, dy = ((torch.rand(tokens, d, generator=g, device="cuda") * spread(d)).to(dt) for _ in range(2))
    h = torch.rand(tokens, rank, generator=g, device="cuda") * spread(rank)
    A, B = (torch.rand(1, *s, generator=g, device="cuda").to(dt) for s in ((rank, d), (d, rank)))
    scale = 2.0 ** -16
    batch = AD.Batch(ctx, [0, tokens], [0], [rank], rank, [scale])
    work = batch.workspace(d, d, dt)
    dx, dA, dB = torch.empty_like(x), torch.empty_like(A), torch.empty_like(B)
    batch.backward(x, h, dy, A, B, dx, dA, dB, work=work, stream=torch.cuda.current_stream())
    want_A = torch.zeros(rank, d, dtype=torch.float64, device="cuda")
    want_B = torch.zeros(d, rank, dtype=torch.float64, device="cuda")
    for k in range(0, tokens, 1 << 20):
        t = slice(k, k + (1 << 20))
        y = dy[t].double()
        want_A += (scale * (y @ B[0].double())).T @ x[t].double()
        want_B += scale * (y.T @ h[t].double())
    assert ctx.device_check() == F.FIONA_OK
    assert float(want_A.max()) < 60000 and float(want_B.max()) < 60000  # (fp16's range)
    bound = CHAIN + rounding_mean(UNIT[dtype], d * rank)
    # (dh is a short chain of its own)
    off = mean_off(dA[0], want_A), mean_off(dB[0], want_B)
    assert off[0] <= bound + CHAIN and off[1] <= bound, off


@pytest.mark.parametrize("rank", [8, 72])
def test_hidden_values_of_a_very_wide_layer(ctx, rank):
    """As many token tiles as there are resident blocks, so that none of them is
    cut along the columns but to bound its chains."""
    n, d_in, d_out = 320, 1 << 20, 64
    g = torch.Generator(device="cuda").manual_seed(rank)
    x = torch.rand(n, d_in, generator=g, device="cuda")  # (rows that spread over an octave)
    x = (x * (torch.rand(n, 1, generator=g, device="cuda") + 1)).bfloat16()
    A = torch.rand(2, rank, d_in, generator=g, device="cuda").bfloat16()
    B = torch.rand(2, d_out, rank, generator=g, device="cuda").bfloat16()
    batch = AD.Batch(ctx, list(range(n + 1)), [i % 2 for i in range(n)], [rank] * 2, rank)
    out, h = torch.empty(n, d_out, dtype=x.dtype, device="cuda"), torch.empty(n, rank, device="cuda")
    batch.forward(x, A, B, out, h=h, work=batch.workspace(d_in, d_out, x.dtype), stream=torch.cuda.current_stream())
    want = torch.empty(n, rank, dtype=torch.float64, device="cuda")
    for i in range(2):
        want[i::2] = x[i::2].double() @ A[i].double().T
    assert ctx.device_check() == F.FIONA_OK
    assert mean_off(h, want) <= CHAIN, mean_off(h, want)
    want = torch.stack([want[i] @ B[i % 2].double().T for i in range(n)])
    off = mean_off(out, want)
    assert off <= 2 * CHAIN + rounding_mean(UNIT["bf16"], out.numel()), off
