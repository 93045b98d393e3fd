"""The adapters and the dropout by their formulas in 64 bits (numpy), with the
sums of absolute terms that bound the rounding of a 32-bit evaluation."""
import numpy as np

from paper_2609_35352_gb300 import workloads as W

# unit roundoffs: half the spacing at 1
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# smallest positive value (an output below it is lost whole)
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}
DROPOUT_STREAM = 4


def keep_mask(rows, cols, p, seed, offset):
    groups = (cols + 3) // 4
    key = W.stream_key(seed & W.MASK64, DROPOUT_STREAM)
    n = np.arange(rows * groups, dtype=np.uint64) + np.uint64(offset & W.MASK64)
    v = W.raw64_np(key, n).reshape(rows, groups, 1)
    fields = (v >> (np.arange(4, dtype=np.uint64) * np.uint64(16))) & np.uint64(0xFFFF)
    return fields.reshape(rows, groups * 4)[:, :cols] >= np.uint64(round(p * 65536))


def factor_of(p):
    level = round(p * 65536)
    return 65536.0 / (65536 - level) if level < 65536 else 0.0


class Reference:
    """Inputs as float64 arrays (exactly the kernels' values); drop = (p, seed,
    offset) or None.  Every result comes with the sum of its absolute terms."""

    def __init__(self, starts, ids, ranks, scales, r_max, x, A, B, drop=None):
        self.starts, self.ids, self.ranks, self.r_max = starts, ids, ranks, r_max
        self.scales = [1.0] * len(ranks) if scales is None else [float(np.float32(s)) for s in scales]
        self.A, self.B = A, B
        self.keep = np.ones(x.shape, bool)
        self.factor = 1.0
        if drop is not None:
            self.keep = keep_mask(x.shape[0], x.shape[1], *drop)
            self.factor = factor_of(drop[0])
        self.x = np.where(self.keep, x, 0.0) * self.factor if self.factor else np.zeros_like(x)

    def spans(self):
        for b, e, a in zip(self.starts, self.starts[1:], self.ids):
            if a >= 0 and e > b:
                yield slice(b, e), a, self.ranks[a], self.scales[a]

    def hidden(self):
        h = np.zeros((self.x.shape[0], self.r_max))
        m = np.zeros_like(h)
        for t, a, k, _ in self.spans():
            h[t, :k] = self.x[t] @ self.A[a, :k].T
            m[t, :k] = np.abs(self.x[t]) @ np.abs(self.A[a, :k]).T
        return h, m

    def forward(self, base):
        h, hm = self.hidden()
        out = np.zeros((self.x.shape[0], self.B.shape[1])) if base is None else base.copy()
        m = np.abs(out)
        for t, a, k, s in self.spans():
            out[t] += s * (h[t, :k] @ self.B[a, :, :k].T)
            m[t] += abs(s) * (hm[t, :k] @ np.abs(self.B[a, :, :k]).T)
        return out, m

    def backward(self, h, dy, dx_base=None):
        dx = np.zeros_like(self.x) if dx_base is None else dx_base.copy()
        mx = np.abs(dx)
        dA, dB = np.zeros_like(self.A), np.zeros_like(self.B)
        mA, mB = np.zeros_like(dA), np.zeros_like(dB)
        for t, a, k, s in self.spans():
            dh, m = s * (dy[t] @ self.B[a, :, :k]), abs(s) * (np.abs(dy[t]) @ np.abs(self.B[a, :, :k]))
            d = self.factor * np.where(self.keep[t], 1.0, 0.0)
            dx[t] += d * (dh @ self.A[a, :k])
            mx[t] += d * (m @ np.abs(self.A[a, :k]))
            dA[a, :k] += dh.T @ self.x[t]
            mA[a, :k] += m.T @ np.abs(self.x[t])
            dB[a, :, :k] += s * (dy[t].T @ h[t, :k])
            mB[a, :, :k] += abs(s) * (np.abs(dy[t]).T @ np.abs(h[t, :k]))
        return (dx, mx), (dA, mA), (dB, mB)


def allowed(dtype, value, terms, n, split=True):
    """How far a result may be off: an fp32 sum of n terms in any order (each
    product, addition and factor rounds once: n + 8 roundings of 2^-24, and an
    accumulator that cuts instead of rounding errs by twice as much), an operand
    in two 16-bit parts (2^-16 of every term; none in fp32), and the last rounding
    to the type.  Splitting fp16 goes by a power of two for many values at once: the
    floor of 2^-30 of the largest sum."""
    bound = terms * (2 * (n + 8) * 2.0 ** -24)
    if split and dtype != "f32":
        bound = bound + terms * 2.0 ** -16
        if dtype == "f16" and terms.size:
            bound = bound + terms.max() * 2.0 ** -30
    return bound * (1 + UNIT[dtype]) + UNIT[dtype] * np.abs(value) + TINY[dtype]


def check(name, dtype, got, value, terms, n, split=True):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == value.shape, name
    off = np.abs(got - value)
    bad = ~(off <= allowed(dtype, value, terms, n, split))
    assert not bad.any(), "%s: %d of %d off, first at %s: %r, not %r" % (
        name, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), got[bad][0], value[bad][0])
