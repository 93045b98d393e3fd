"""What the adapters' binding checks before it passes addresses on (no GPU: a
validation-only context whose tensors are taken to be the host's)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_35352_gb300 import adapters as AD
from paper_2609_35352_gb300 import build as B
from paper_2609_35352_gb300 import fiona as F
from paper_2609_35352_gb300 import workloads as W

T, D_IN, D_OUT, R = 6, 16, 24, 8


@pytest.fixture(scope="module")
def ctx():
    B.build()
    return F.Context(1024, W.ntt_primes(1024, 40, 1), device=F.FIONA_DEVICE_NONE)


@pytest.fixture
def batch(ctx):
    b = AD.Batch(ctx, [0, T], [0], [R], R)
    b._dev = torch.device("cpu")
    return b


def aligned(*shape, dtype=torch.bfloat16):
    t = torch.zeros(shape, dtype=dtype)
    assert t.data_ptr() % 16 == 0
    return t


def call(batch, backward, work):
    x, out = aligned(T, D_IN), aligned(T, D_OUT)
    A, B_ = aligned(1, R, D_IN), aligned(1, D_OUT, R)
    h = aligned(T, R, dtype=torch.float32)
    if backward:
        batch.backward(x, h, out, A, B_, aligned(T, D_IN), torch.zeros_like(A), torch.zeros_like(B_), work=work)
    else:
        batch.forward(x, A, B_, out, h=h, work=work)


@pytest.mark.parametrize("backward", [False, True])
def test_workspaces(batch, backward):
    n = batch.work_bytes(D_IN, D_OUT, torch.bfloat16)
    with pytest.raises(F.FionaError) as e:  # all is well but for the device
        call(batch, backward, aligned(n, dtype=torch.uint8))
    assert e.value.status == F.FIONA_ERR_NODEVICE
    with pytest.raises(ValueError, match="workspace"):
        call(batch, backward, None)
    with pytest.raises(ValueError, match="workspace"):  # another device's
        call(batch, backward, torch.empty(n, dtype=torch.uint8, device="meta"))
    with pytest.raises(ValueError, match="workspace"):  # every other byte of a buffer
        call(batch, backward, aligned(2 * n, dtype=torch.uint8)[::2])
    batch._dev = torch.device("meta")
    with pytest.raises(ValueError):
        call(batch, backward, aligned(n, dtype=torch.uint8))


def test_indices_are_taken_as_they_are(ctx):
    """Whole numbers that the C arrays cannot hold are refused, not wrapped or cut."""
    import numpy as np
    good = dict(starts=[0, 3, 5], adapters=[0, -1], ranks=[4, 8], r_max=8)
    AD.Batch(ctx, **good)
    AD.Batch(ctx, **{k: np.array(v) if k != "r_max" else v for k, v in good.items()})
    AD.Batch(ctx, np.array([0.0, 3.0, 5.0]), [0, -1], torch.tensor([4, 8]), 8)
    AD.Batch(ctx, [0], [], [], 8)
    for change in (dict(adapters=np.array([1 << 32, -1])), dict(adapters=[0.5, -1]), dict(ranks=np.array([(1 << 32) + 4, 8])),
                   dict(ranks=np.array([4, -(1 << 32)])), dict(starts=np.array([0, 3.5, 5])), dict(starts=[0, float("nan"), 5]),
                   dict(starts=[0, -1, 5]), dict(adapters=[1 << 40, -1]), dict(ranks=np.array([2.0 ** 33, 8])), dict(adapters=[float(1 << 31), -1]),
                   dict(starts=[0, 2.0 ** 64, 5]), dict(r_max=-1), dict(r_max=(1 << 32) + 8), dict(r_max=float("nan")), dict(ranks=["a", 8]), dict(r_max=8.5)):
        with pytest.raises(ValueError):
            AD.Batch(ctx, **dict(good, **change))
