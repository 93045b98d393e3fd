"""Adapter inputs whose results are known to the last bit: small integers (and
scales and a dropout factor that are powers of two), so that every product and
every partial sum is exact in 32 bits in any order, in operands of 16 bits in two
parts too, and an output is the exact sum rounded once to its type."""
import numpy as np

from adapter_util import Reference

# significand bits of a type
BITS = {"f32": 24, "f16": 11, "bf16": 8}


def round_to(dtype, v):
    """v (float64) to the nearest value of the type, ties to even (as float64)."""
    if dtype == "f16":
        with np.errstate(over="ignore"):  # (past its range: infinite, in the kernels too)
            return v.astype(np.float16).astype(np.float64)
    f = v.astype(np.float32)
    if dtype == "f32":
        return f.astype(np.float64)
    u = f.view(np.uint32)
    u = (u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)
    return u.view(np.float32).astype(np.float64)


class Integers:
    """x, A, B, dy, h and the bases of a batch, as float64 arrays."""

    def __init__(self, starts, ids, ranks, r_max, d_in, d_out, p=0.0, seed=0):
        rng = np.random.default_rng(seed)
        T, n = starts[-1], len(ranks)
        self.starts, self.ids, self.ranks, self.r_max = starts, ids, ranks, r_max
        # (fp16's range: sums of some 10^6 times 2^-6)
        self.scales = [2.0 ** -(5 + a % 3) for a in range(n)]
        self.drop = (0.5, 11 + seed, 1 << 33) if p else None

        def ints(most, *shape, density=1.0):
            v = rng.integers(-most, most + 1, shape).astype(np.float64)
            return v if density == 1.0 else np.where(rng.random(shape) < density, v, 0.0)

        self.x = ints(2, T, d_in, density=0.1 if d_in > 16 else 1.0)
        self.A, self.B = ints(31, n, r_max, d_in), ints(127, n, d_out, r_max)
        self.dy = ints(3, T, d_out)
        self.h = ints(8191, T, r_max, density=0.25)
        for b, e, a in zip(starts, starts[1:], ids):  # zero at and above the rank
            self.h[b:e, ranks[a] if a >= 0 else 0:] = 0.0
        self.base, self.dx_base = ints(100, T, d_out), ints(100, T, d_in)
        self.ref = Reference(starts, ids, ranks, self.scales, r_max, self.x, self.A, self.B, self.drop)
        self._check()

    def _check(self):
        """That all of it is exact: sums of absolute terms below 2^24, in units of the
        smallest scale where one is applied before; h and dh of at most 16 bits."""
        ref, unit = self.ref, 2.0 ** -7
        assert not ref.x.size or np.abs(ref.hidden()[0]).max(initial=0) < 2 ** 16
        for t, a, k, s in ref.spans():
            h, dh = np.abs(ref.x[t]) @ np.abs(self.A[a, :k]).T, self.dy[t] @ self.B[a, :, :k]
            assert (np.abs(self.dy[t]) @ np.abs(self.B[a, :, :k])).max(initial=0) < 2 ** 24
            assert np.abs(dh).max(initial=0) < 2 ** 16
            assert (np.abs(ref.hidden()[0][t, :k]) @ np.abs(self.B[a, :, :k]).T).max(initial=0) + 100 / unit < 2 ** 24
            assert h.max(initial=0) < 2 ** 24
            assert 2 * (np.abs(dh) @ np.abs(self.A[a, :k])).max(initial=0) + 100 / unit < 2 ** 24
        for a in range(len(self.ranks)):
            rows = np.concatenate([np.arange(t.start, t.stop) for t, b, _, _ in ref.spans() if b == a] or [np.arange(0)])
            dh = np.abs(self.dy[rows] @ self.B[a])
            assert (dh.T @ np.abs(ref.x[rows])).max(initial=0) < 2 ** 24
            assert (np.abs(self.dy[rows]).T @ np.abs(self.h[rows])).max(initial=0) < 2 ** 24

    def forward(self):
        return self.ref.forward(self.base)[0], self.ref.hidden()[0]

    def backward(self, dh_of=lambda v: v, h_of=lambda v: v, skip=None):
        """dx, dA and dB; `dh_of`, `h_of`: what becomes of an operand; `skip`: a token
        left out of the sums (mistakes that a test has to see)."""
        ref, dx = self.ref, self.dx_base.copy()
        dA, dB = np.zeros_like(self.A), np.zeros_like(self.B)
        for t, a, k, s in ref.spans():
            dh = dh_of(s * (self.dy[t] @ self.B[a, :, :k]))
            dx[t] += ref.factor * np.where(ref.keep[t], dh @ self.A[a, :k], 0.0)
            live = np.arange(t.start, t.stop) != skip
            dA[a, :k] += dh[live].T @ ref.x[t][live]
            dB[a, :, :k] += s * (self.dy[t][live].T @ h_of(self.h[t][live][:, :k]))
        return dx, dA, dB
