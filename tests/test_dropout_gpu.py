"""Dropout with a mask that is never stored, against its definition: the kept
elements exactly, and every value to one rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

from adapter_util import TINY, UNIT, factor_of, keep_mask  # noqa: E402

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


def make(rows, cols, dtype, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(rows, cols + pad, generator=g, device="cuda").to(DT[dtype])
    return t[:, pad // 2:pad // 2 + cols]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 5, 0), (17, 64, 0), (300, 777, 0), (64, 1024, 0),
                                           (33, 256, 2), (33, 250, 8), (5, 4099, 3), (2, 65536, 0)])
def test_against_the_definition(ctx, dtype, p, rows, cols, pad):
    x, res = make(rows, cols, dtype, pad, 1), make(rows, cols, dtype, pad, 2)
    out = make(rows, cols, dtype, pad, 3)
    drop = AD.Dropout(p, 2609 + cols, (1 << 50) + rows)
    keep = keep_mask(rows, cols, p, drop.seed, drop.offset)
    value = np.where(keep, x.double().cpu().numpy() * factor_of(p), 0.0)
    r = res.double().cpu().numpy()
    for residual in (None, res):
        AD.dropout(ctx, x, out, drop, residual=residual)
        torch.cuda.synchronize()
        got = out.double().cpu().numpy()
        want = value if residual is None else value + r
        # the factor, the product and the sum round in fp32, the result in its type
        size = np.abs(value) + (0 if residual is None else np.abs(r))
        assert (np.abs(got - want) <= UNIT[dtype] * np.abs(want) + 4 * 2.0 ** -24 * size + TINY[dtype]).all()
        if residual is None:
            assert (got[~keep] == 0).all()
            # (a kept value below the type's smallest is the only one that may vanish)
            assert ((got != 0) == (keep & (np.abs(value) >= TINY[dtype]))).all()
        else:
            assert np.array_equal(got[~keep], r[~keep])
    dx = make(rows, cols, dtype, pad, 4)
    AD.dropout_backward(ctx, x, dx, drop)
    AD.dropout(ctx, x, out, drop)
    assert torch.equal(dx, out)


def test_in_place_and_neighbours(ctx):
    """out may be x or residual; columns beside a strided range stay."""
    for dtype in DT:
        x, res = make(40, 100, dtype, 0, 1), make(40, 100, dtype, 0, 2)
        drop = AD.Dropout(0.4, 5)
        want = torch.empty_like(x)
        AD.dropout(ctx, x, want, drop, residual=res)
        a, b = x.clone(), res.clone()
        AD.dropout(ctx, a, a, drop, residual=res)
        AD.dropout(ctx, x, b, drop, residual=b)
        assert torch.equal(a, want) and torch.equal(b, want)
        wide = torch.full((40, 128), 3.0, dtype=DT[dtype], device="cuda")
        AD.dropout(ctx, x, wide[:, 9:109], drop, residual=res)
        assert torch.equal(wide[:, 9:109], want)
        assert (wide[:, :9] == 3).all() and (wide[:, 109:] == 3).all()


def test_dropped_values_are_zero_whatever_they_held(ctx):
    for dtype in DT:
        x = torch.full((8, 512), float("nan"), dtype=DT[dtype], device="cuda")
        x[1::2] = float("inf")
        out = torch.empty_like(x)
        AD.dropout(ctx, x, out, AD.Dropout(0.5, 3))
        keep = torch.from_numpy(keep_mask(8, 512, 0.5, 3, 0)).cuda()
        assert (out[~keep] == 0).all() and not torch.isfinite(out[keep]).any()
        AD.dropout(ctx, x, out, AD.Dropout(1.0, 3))
        assert (out == 0).all()


def test_offsets_continue_a_mask(ctx):
    """Rows t and on of a mask are the mask at the offset that `advance` gives,
    also past 32 bits; other seeds give other masks."""
    x = make(64, 333, "f32")
    whole, part = torch.empty_like(x), torch.empty_like(x[40:])
    for offset in (0, (1 << 32) - 7, (1 << 64) - 100):
        drop = AD.Dropout(0.3, 11, offset)
        AD.dropout(ctx, x, whole, drop)
        AD.dropout(ctx, x[40:], part, drop.advance(40, 333))
        assert torch.equal(whole[40:], part)
    other = torch.empty_like(x)
    AD.dropout(ctx, x, other, AD.Dropout(0.3, 12, offset))
    assert not torch.equal(whole == 0, other == 0)


def test_share_of_kept_elements(ctx):
    """About 1 - p of the elements stay: within six standard deviations, per
    column field and in all."""
    x = torch.ones(4096, 1024, device="cuda")
    out = torch.empty_like(x)
    for p in (0.05, 0.5, 0.9):
        AD.dropout(ctx, x, out, AD.Dropout(p, 1234))
        kept = (out != 0).double()
        for part in (kept, kept[:, 0::4], kept[:, 1::4], kept[:, 2::4], kept[:, 3::4]):
            assert abs(float(part.mean()) - (1 - p)) < 6 * (p * (1 - p) / part.numel()) ** 0.5 + 2.0 ** -17


def test_many_rows(ctx):
    """Element offsets past 32 bits."""
    rows, cols = 70000, 65000
    x = torch.ones(1, cols, dtype=torch.float16, device="cuda").expand(rows, cols)
    out = torch.empty(rows, cols, dtype=torch.float16, device="cuda")
    drop = AD.Dropout(0.5, 21)
    AD.dropout(ctx, x, out, drop)
    tail = torch.empty(50, cols, dtype=torch.float16, device="cuda")
    AD.dropout(ctx, x[:50], tail, drop.advance(rows - 50, cols))
    assert torch.equal(out[-50:], tail)
    keep = keep_mask(50, cols, 0.5, 21, (rows - 50) * (cols // 4))
    assert np.array_equal(tail.cpu().numpy() != 0, keep)


def test_other_stream(ctx):
    x = make(512, 512, "bf16")
    out, want = torch.empty_like(x), torch.empty_like(x)
    drop = AD.Dropout(0.2, 8)
    AD.dropout(ctx, x, want, drop)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    AD.dropout(ctx, x, out, drop, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
