"""Waits of the rows kernel that run out in many clusters at once: every CTA ends,
none while another may still write to its shared memory, and the context goes on."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

from test_adapters_gpu import Problem  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,adapters", [(300, 300), (300, 80)])
def test_many_clusters_that_give_up(ctx, dtype, n, adapters, monkeypatch):
    starts, ids, ranks = list(range(n + 1)), [i * 7 % adapters for i in range(n)], [16] * adapters
    monkeypatch.setenv("FIONA_ADAPTER_TEST_STALL", "1")
    stalled = Problem(ctx, dtype, starts, ids, ranks, 16, 512, 384)
    monkeypatch.delenv("FIONA_ADAPTER_TEST_STALL")
    assert ctx.device_check() == F.FIONA_OK
    stalled.forward()
    assert ctx.device_check() == F.FIONA_ERR_TIMEOUT
    good = Problem(ctx, dtype, starts, ids, ranks, 16, 512, 384)
    good.forward()
    torch.cuda.synchronize()
    good.check_forward()
    assert ctx.device_check() == F.FIONA_OK
