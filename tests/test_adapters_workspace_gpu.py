"""A call stays within the workspace that it asks for: bytes behind it keep what they
held, whichever kernels run and however the gradients are added up."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

from test_adapters_gpu import DT, Problem  # noqa: E402

GUARD = 4 << 20


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("starts,ids,ranks,r_max,d_in,d_out", [
    (list(range(65)), [i % 48 for i in range(64)], [16] * 50, 16, 1024, 512),     # one chunk an adapter, two without rows
    ([0, 130, 400, 401], [0, 1, 2], [128, 90, 128], 128, 512, 264),               # the same, above rank 64
    ([0, 5000, 5600], [0, 1], [32, 7], 32, 768, 640),                             # chunks that are added up
    ([0, 3000, 3500], [0, 1], [72, 128], 128, 256, 512),
    ([0, 1800, 1803, 1900, 3000], [0, 1, -1, 2], [43, 41, 7], 43, 1001, 777),      # sizes off eight
    ([0, 9, 40], [0, 1], [3, 5], 5, 77, 131),
    ([0, 0], [0], [8], 8, 64, 64),
])
def test_nothing_behind_the_workspace_changes(ctx, dtype, starts, ids, ranks, r_max, d_in, d_out):
    pr = Problem(ctx, dtype, starts, ids, ranks, r_max, d_in, d_out, seed=d_in, p=0.1)
    n = pr.batch.work_bytes(d_in, d_out, DT[dtype])
    whole = torch.full((n + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    pr.work = whole[:n] if n else whole
    pr.run_and_check()
    assert bool((whole[n:] == 0xA5).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("starts,ids,r_max,d_in,d_out", [
    (list(range(65)), [i % 48 for i in range(64)], 16, 1024, 512), ([0, 700, 701, 2000], [0, 1, 0], 24, 768, 640),
    (list(range(41)), [i % 3 - 1 for i in range(40)], 8, 200000, 64), ([0, 3000, 3500], [0, -1], 128, 256, 512),
    ([0, 1800, 1803, 1900, 3000], [0, 1, -1, 2], 43, 1001, 777), ([0, 9, 40], [0, 1], 5, 77, 131)])
def test_forward_only(ctx, dtype, starts, ids, r_max, d_in, d_out):
    pr = Problem(ctx, dtype, starts, ids, [r_max] * (max(ids) + 1), r_max, d_in, d_out, seed=d_out)
    pr.batch = AD.Batch(ctx, starts, ids, pr.ranks, r_max, pr.scales, gradients=False)
    n = pr.batch.work_bytes(d_in, d_out, DT[dtype])
    whole = torch.full((n + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    pr.work = whole[:n] if n else whole
    pr.forward()
    torch.cuda.synchronize()
    pr.check_forward()
    assert bool((whole[n:] == 0xA5).all())
    with pytest.raises(F.FionaError):
        pr.backward()
