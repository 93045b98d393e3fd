"""The adapters bit for bit, on integers whose results are known exactly
(adapter_exact.py; test_adapters_exact_host.py says what they can see: a token
left out of a sum, an operand without its second part)."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

from adapter_exact import Integers, round_to  # noqa: E402

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CASES = {
    "short": ([0, 3, 400, 700], [0, 1, 0], [16, 11], 16, 256, 200),
    "long": ([0, 3000, 3001], [1, 0], [16, 16], 16, 512, 640),
    "odd": ([0, 1800, 1803, 1900, 4000], [0, 1, -1, 2], [43, 41, 7], 43, 257, 203),
    "rank 72": ([0, 300, 900, 901], [1, 0, 1], [72, 65], 72, 320, 264),
    "rank 128": ([0, 1500, 2600], [0, 1], [128, 113], 128, 256, 392),
    "tokens": (list(range(41)), [i % 4 - 1 for i in range(40)], [32, 9, 17], 32, 768, 520),
    "one": ([0, 1], [0], [8], 8, 512, 72),
}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_every_bit(ctx, dtype, name, p):
    q, dt = Integers(*CASES[name], p=p), DT[dtype]

    def put(v, t=dt):
        return torch.from_numpy(v).cuda().to(t)

    x, A, B, dy, base, dx_base = (put(v) for v in (q.x, q.A, q.B, q.dy, q.base, q.dx_base))
    h = put(q.h, torch.float32)
    batch = AD.Batch(ctx, q.starts, q.ids, q.ranks, q.r_max, q.scales)
    work = batch.workspace(x.shape[1], base.shape[1], dt)
    out, made, dx, dA, dB = (torch.full_like(t, 7.0) for t in (base, h, x, A, B))
    drop = AD.Dropout(*q.drop) if q.drop else None
    s = torch.cuda.current_stream()
    batch.forward(x, A, B, out, base=base, h=made, dropout=drop, work=work, stream=s)
    batch.backward(x, h, dy, A, B, dx, dA, dB, dx_base=dx_base, dropout=drop, work=work, stream=s)
    torch.cuda.synchronize()
    assert ctx.device_check() == F.FIONA_OK
    want = dict(zip(("out", "h", "dx", "dA", "dB"), q.forward() + q.backward()))
    for key, got in (("out", out), ("h", made), ("dx", dx), ("dA", dA), ("dB", dB)):
        exact = torch.from_numpy(round_to("f32" if key == "h" else dtype, want[key])).cuda()
        bad = got.double() != exact
        assert not bad.any(), "%s: %d of %d, first at %s" % (key, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist())
