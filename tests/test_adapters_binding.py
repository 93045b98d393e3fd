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
