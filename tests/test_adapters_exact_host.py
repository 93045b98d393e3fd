"""What the bit-exact cases (adapter_exact.py) can see: each mistake, planted in
the oracle, has to change rounded gradients."""
import numpy as np
import pytest

from adapter_exact import BITS, Integers, round_to

SMALL = ([0, 3, 400, 700], [0, 1, 0], [16, 11], 16, 256, 200)
# (those of the GPU tests)
LONG = ([0, 3000, 3001], [1, 0], [16, 16], 16, 512, 640)
ODD = ([0, 1800, 1803, 1900, 4000], [0, 1, -1, 2], [43, 41, 7], 43, 257, 203)


def changed(dtype, good, bad):
    return float(np.mean(round_to(dtype, good) != round_to(dtype, bad)))


@pytest.mark.parametrize("case", [SMALL, LONG, ODD])
def test_formulas_agree(case):
    """The integer oracle against the tests' other one."""
    q = Integers(*case, p=0.5)
    (dx, _), (dA, _), (dB, _) = q.ref.backward(q.h, q.dy, q.dx_base)
    for a, b in zip(q.backward(), (dx, dA, dB)):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", [SMALL, LONG, ODD])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_mistakes_are_seen(dtype, case, p):
    q = Integers(*case, p=p)
    _, dA, dB = q.backward()
    adapter = case[1][-1] if case is not LONG else 1
    token = case[0][1] - 1 if case is LONG else case[0][-1] - 1
    _, lost_A, lost_B = q.backward(skip=token)
    # (a token has a tenth of its x, the half of them kept, and a quarter of its h;
    # in 8 bits its part is below half a unit of most sums)
    share = {"f32": 0.02, "f16": 0.01, "bf16": 0.002}[dtype]
    k = q.ranks[adapter]
    assert changed(dtype, dA[adapter, :k], lost_A[adapter, :k]) > share
    assert changed(dtype, dB[adapter, :, :k], lost_B[adapter, :, :k]) > share
    if dtype == "f32":
        return
    half = lambda v: round_to(dtype, v)  # noqa: E731  (one part of 8 or 11 bits)
    dx1, hi_A, hi_B = q.backward(dh_of=half, h_of=half)
    assert changed(dtype, dA, hi_A) > 0.01 and changed(dtype, dB, hi_B) > 0.01
    assert changed(dtype, q.backward()[0], dx1) > 0.01


def test_round_to():
    v = np.array([257.0, 258.0, 259.0, 2049.0, 2051.0, -1.0, 0.0])
    assert round_to("bf16", v).tolist() == [256.0, 258.0, 260.0, 2048.0, 2048.0, -1.0, 0.0]
    assert round_to("f16", v).tolist() == [257.0, 258.0, 259.0, 2048.0, 2052.0, -1.0, 0.0]
    assert BITS["f32"] == 24 and round_to("f32", np.array([16777217.0]))[0] == 16777216.0
