"""The layer norm by its formulas in 64 bits (numpy), with bounds of the rounding of a
32-bit evaluation.  u = 2^-24 is a rounding in fp32; a sum of n terms in any order of at
most `chain` additions one after another errs by chain u times the terms' absolute sum."""
import numpy as np

from adapter_util import TINY, UNIT, factor_of, keep_mask

U = 2.0 ** -24


def chain_of(cols):
    """Additions one after another in a row's sum: a thread's share of the columns, then
    a tree over the threads."""
    return cols / 256 + 64


def column_chain_of(rows):
    """Those in a column's sum: at most 512 rows, then the runs' sums, then a tree."""
    return min(rows, 512) + rows / (512 * 32) + 64


def forward(x, res, weight, bias, eps, drop=None):
    """Inputs as float64 arrays; drop = (p, seed, offset) or None.  A dict of (value, bound
    before the last rounding)."""
    xf = x
    if drop is not None:
        xf = np.where(keep_mask(x.shape[0], x.shape[1], *drop), x, 0.0) * factor_of(drop[0])
    s = xf if res is None else xf + res
    n = chain_of(x.shape[1])
    ds = 3 * U * np.abs(xf) + U * np.abs(s)
    mean = s.mean(1, keepdims=True)
    d = s - mean
    var = (d * d).mean(1, keepdims=True)
    r = 1 / np.sqrt(var + eps)
    # the first mean is off by n u avg|s|; taking out what it left, n u of that stays
    off = n * U * np.abs(s).mean(1, keepdims=True)
    dmean = ds.mean(1, keepdims=True) + n * U * (np.abs(d).mean(1, keepdims=True) + off)
    dd = ds + dmean + 3 * U * (np.abs(d) + off)
    dvar = (2 * np.abs(d) * dd + dd * dd).mean(1, keepdims=True) + (n + 4) * U * (var + off * off)
    share = dvar / (2 * (var + eps)) + 4 * U
    dr = r * share * np.where(share > 0.1, 4.0, 1.2)  # (second order)
    w = 1.0 if weight is None else weight
    y = w * d * r + (0.0 if bias is None else bias)
    dy = np.abs(w) * (dd * (r + dr) + np.abs(d) * dr) + 4 * U * (np.abs(w * d * r) + np.abs(y))
    return {"out": (y, dy), "sum": (s, ds), "mean": (mean[:, 0], (dmean + U * np.abs(mean))[:, 0]), "rstd": (r[:, 0], dr[:, 0])}


def backward(dy, s, mean, rstd, weight=None, dsum=None, drop=None):
    rows, cols = dy.shape
    n, c = chain_of(cols), column_chain_of(rows)
    mean, r = mean[:, None], rstd[:, None]
    xh = (s - mean) * r
    g = dy if weight is None else dy * weight
    a, b = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    da, db = (n + 3) * U * np.abs(g).mean(1, keepdims=True), (n + 6) * U * np.abs(g * xh).mean(1, keepdims=True)
    ds = r * (g - a - xh * b)
    dds = np.abs(r) * (da + np.abs(xh) * db + 6 * U * (np.abs(g) + np.abs(a) + np.abs(xh * b)))
    if dsum is not None:
        ds = ds + dsum
        dds = dds + U * np.abs(ds)
    dx, ddx = ds, dds
    if drop is not None:
        f = np.where(keep_mask(rows, cols, *drop), factor_of(drop[0]), 0.0)
        dx, ddx = ds * f, dds * f + 3 * U * np.abs(ds * f)
    return {"dresidual": (ds, dds), "dx": (dx, ddx), "dweight": ((dy * xh).sum(0), (c + 5) * U * np.abs(dy * xh).sum(0)),
            "dbias": (dy.sum(0), (c + 1) * U * np.abs(dy).sum(0))}


def check(name, dtype, got, value, bound):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == value.shape, name
    allowed = bound * (1 + UNIT[dtype]) * 1.01 + UNIT[dtype] * np.abs(value) + TINY[dtype]
    bad = ~(np.abs(got - value) <= allowed)
    assert not bad.any(), "%s: %d of %d off, first at %s: %r, not %r (allowed %.3g)" % (
        name, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), got[bad][0], value[bad][0], allowed[bad][0])
