"""AdamW by its formulas in 64 bits (numpy), with bounds of the rounding of a 32-bit
evaluation (u = 2^-24 a rounding in fp32)."""
import numpy as np

from adapter_util import TINY, UNIT

U = 2.0 ** -24
BLOCK = 256


def places(counts):
    padded = -(-np.asarray(counts, dtype=np.int64) // BLOCK) * BLOCK
    return np.cumsum(padded) - padded, int(padded.sum())


def decode_m(q, scale):
    q = np.asarray(q, dtype=np.float64)
    return q * np.abs(q) / 127 ** 2 * scale


def decode_v(q, scale):
    return (np.asarray(q, dtype=np.float64) ** 2 / 255 ** 2 * scale) ** 2


class Group:
    def __init__(self, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_norm=np.inf):
        self.lr, self.beta1, self.beta2, self.eps = float(np.float32(lr)), beta1, beta2, eps
        self.weight_decay, self.max_norm = weight_decay, max_norm


def norm_of(grads):
    return float(np.sqrt(sum((g * g).sum() for g in grads)))


def step(group, t, w, m, v, g, norm=None):
    """A tensor's new weights and moments (t: the step count after the step), each with
    the bound of its rounding in fp32.  norm: the group's, where it is taken."""
    k = group.max_norm / norm if norm is not None and norm > group.max_norm else 1.0
    # a norm: sums of squares by lanes of 32 elements, a tree, then fp64; a quotient
    dk = 60 * U if k != 1.0 else 0.0
    b1, b2 = group.beta1, group.beta2
    g = g * k
    dg = (dk + 2 * U) * np.abs(g)
    m1 = b1 * m + (1 - b1) * g
    dm = 3 * U * (b1 * np.abs(m) + (1 - b1) * np.abs(g)) + (1 - b1) * dg
    v1 = b2 * v + (1 - b2) * g * g
    dv = 4 * U * v1 + (1 - b2) * 2 * np.abs(g) * dg + 2.0 ** -149
    c1, c2 = 1 - b1 ** t, 1 - b2 ** t
    root = np.sqrt(v1 / c2)
    den = root + group.eps
    # (the root's error is dv / (2 root), or its own size where v is of the order of dv)
    droot = np.minimum(dv / c2 / np.maximum(root, 1e-300), np.sqrt(2 * dv / c2)) + 4 * U * root
    step_ = group.lr * (m1 / c1) / den
    dstep = group.lr * (dm / c1) / den + np.abs(step_) * (droot / np.maximum(den - droot, 0.1 * den) + 10 * U)
    decay = group.lr * group.weight_decay * w
    w1 = w - decay - step_
    dw = dstep + 4 * U * (np.abs(decay) + np.abs(step_)) + U * np.abs(w1)
    return (w1, dw), (m1, dm), (v1, dv)


def check(name, dtype, got, value, bound):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == value.shape, name
    allowed = bound * (1 + UNIT[dtype]) * 1.01 + UNIT[dtype] * np.abs(value) + TINY[dtype]
    bad = ~(np.abs(got - value) <= allowed)
    assert not bad.any(), "%s: %d of %d off, first at %s: %r, not %r (allowed %.3g)" % (
        name, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), got[bad][0], value[bad][0], allowed[bad][0])


def check_codes(name, codes, scales, value, bound, top):
    """Codes and scales of whole blocks [blocks][256] against the values (m, or u = sqrt v)
    that they were made from: the scale is the block's largest, and a code stands for the
    nearest of q^2 / top^2 of it (half a step), a value above zero of u for 1 at least."""
    codes, value = np.asarray(codes, dtype=np.float64).reshape(-1, BLOCK), value.reshape(-1, BLOCK)
    bound = np.broadcast_to(bound, np.asarray(bound).shape).reshape(-1, BLOCK)
    scales = np.asarray(scales, dtype=np.float64).reshape(-1, 1)
    most, room = np.abs(value).max(1, keepdims=True), bound.max(1, keepdims=True) + 4 * U * np.abs(value).max(1, keepdims=True)
    assert (np.abs(scales - most) <= room + 2.0 ** -100).all(), name + ": scales"
    got = codes * np.abs(codes) / top ** 2 * scales
    q = np.abs(codes)
    half = (2 * q + 1) / 2 / top ** 2 * scales
    off = np.abs(got - value)
    bad = ~(off <= half * (1 + 1e-5) + 2 * room + 2.0 ** -100)
    assert not bad.any(), "%s: %d of %d codes, first at %s: %r for %r of %r" % (
        name, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), codes[bad][0], value[bad][0], scales[np.argwhere(bad)[0][0]])
    assert (np.abs(codes) <= top).all()
    if top == 255:
        assert ((codes >= 1) | (value <= 2 * room) | (scales == 0)).all(), name + ": u above zero with code 0"
