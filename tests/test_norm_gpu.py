"""Layer norm with dropout and residual, and its gradient, against the formulas in 64
bits (norm_util.py derives what rounding may do)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import layernorm as LN  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

import norm_util as NU  # noqa: E402
from adapter_util import keep_mask  # noqa: E402

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SHAPES = [(1, 1, 0), (1, 768, 0), (3, 5, 0), (17, 64, 0), (300, 777, 0), (64, 1024, 0), (33, 256, 2), (33, 250, 8),
          (5, 4099, 3), (2, 65536, 0), (1, 1 << 20, 0), (1000, 8, 0), (2047, 33, 0), (7, 16384, 0), (5, 16392, 0), (130, 2048, 0),
          (40, 8192, 0), (37, 640, 0), (9, 765, 3), (9, 12288, 8), (11, 4096, 0), (10, 511, 1), (700, 264, 0), (3, 32768, 0), (4, 20000, 0), (3, 20001, 0), (300, 16411, 2)]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


def make(rows, cols, dtype, pad=0, seed=0, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = (torch.randn(rows, cols + pad, generator=g, device="cuda") * scale + shift).to(DT[dtype])
    return t[:, pad // 2:pad // 2 + cols]


def vector(cols, dtype, seed, scale=1.0, shift=0.0):
    return make(1, cols, dtype, 0, seed, scale, shift)[0].contiguous()


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def run_forward(ctx, x, res, weight, bias, eps, drop, stream=None):
    rows = x.shape[0]
    r = {"out": torch.empty_strided(x.shape, (max(x.stride(0), x.shape[1]), 1), dtype=x.dtype, device="cuda"),
         "sum": torch.empty(x.shape, dtype=x.dtype, device="cuda"), "mean": torch.empty(rows, device="cuda"),
         "rstd": torch.empty(rows, device="cuda")}
    LN.layer_norm(ctx, x, r["out"], weight=weight, bias=bias, eps=eps, residual=res, dropout=drop, sum=r["sum"], mean=r["mean"],
                  rstd=r["rstd"], stream=stream)
    return r


def check_all(dtype, wtype, got, want):
    for k, (value, bound) in want.items():
        if got.get(k) is not None:
            NU.check(k, "f32" if k in ("mean", "rstd") else wtype if k in ("dweight", "dbias") else dtype, f64(got[k]), value, bound)


def spec(drop):
    return None if drop is None else (drop.p, drop.seed, drop.offset)


@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("rows,cols,pad", SHAPES)
def test_forward(ctx, dtype, wtype, rows, cols, pad):
    x, res = make(rows, cols, dtype, pad, 1), make(rows, cols, dtype, pad, 2, 2.0, 0.5)
    weight, bias = vector(cols, wtype, 3, 0.2, 1.0), vector(cols, wtype, 4)
    for drop, r, w, b in ((AD.Dropout(0.2, 2609 + cols, (1 << 50) + rows), res, weight, bias), (None, None, weight, None), (None, res, None, bias)):
        got = run_forward(ctx, x, r, w, b, 1e-5, drop)
        check_all(dtype, wtype, got, NU.forward(f64(x), f64(r), f64(w), f64(b), 1e-5, spec(drop)))
        plain = torch.empty_like(x)
        LN.layer_norm(ctx, x, plain, weight=w, bias=b, residual=r, dropout=drop)  # (nothing kept)
        assert torch.equal(plain, got["out"])


@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("rows,cols,pad", SHAPES)
def test_backward(ctx, dtype, wtype, rows, cols, pad):
    dy, s, dsum = make(rows, cols, dtype, pad, 1), make(rows, cols, dtype, pad, 2, 2.0, 0.5), make(rows, cols, dtype, pad, 3)
    weight = vector(cols, wtype, 4, 0.2, 1.0)
    mean, rstd = s.double().mean(1).float(), (s.double().var(1, unbiased=False) + 1e-5).rsqrt().float()
    work = LN.workspace(ctx, rows, cols)
    for drop, w, extra in ((AD.Dropout(0.2, 7, 1 << 40), weight, None), (None, weight, dsum), (None, None, None)):
        got = {"dx": torch.empty_like(dy), "dresidual": torch.empty_strided(dy.shape, dy.stride(), dtype=dy.dtype, device="cuda"),
               "dweight": torch.empty(cols, dtype=DT[wtype], device="cuda"), "dbias": torch.empty(cols, dtype=DT[wtype], device="cuda")}
        LN.layer_norm_backward(ctx, dy, s, mean, rstd, weight=w, dsum=extra, dropout=drop, work=work, **got)
        check_all(dtype, wtype, got, NU.backward(f64(dy), f64(s), f64(mean), f64(rstd), f64(w), f64(extra), spec(drop)))
        if drop is None:
            assert torch.equal(got["dx"], got["dresidual"])
        # each output by itself is the same
        for k in got:
            one = torch.empty_like(got[k])
            LN.layer_norm_backward(ctx, dy, s, mean, rstd, weight=w, dsum=extra, dropout=drop, work=work, **{k: one})
            assert torch.equal(one, got[k]), k


def test_random_sizes(ctx):
    rng = np.random.default_rng(2609)
    for i in range(60):
        rows, cols = int(np.exp(rng.uniform(0, 7))), int(np.exp(rng.uniform(0, 9.3)))
        dtype, pad = ["f32", "f16", "bf16"][i % 3], int(rng.integers(0, 9))
        wtype = dtype if rng.random() < 0.5 else "f32"
        drop = AD.Dropout(float(rng.choice([0.1, 0.5])), i, i << 33) if rng.random() < 0.5 else None
        x, res = make(rows, cols, dtype, pad, i), make(rows, cols, dtype, 0, i + 1000, 3.0) if rng.random() < 0.5 else None
        weight, bias = vector(cols, wtype, i + 1, 0.2, 1.0), vector(cols, wtype, i + 2)
        got = run_forward(ctx, x, res, weight, bias, 1e-6, drop)
        check_all(dtype, wtype, got, NU.forward(f64(x), f64(res), f64(weight), f64(bias), 1e-6, spec(drop)))
        dy = make(rows, cols, dtype, pad, i + 3)
        g = {"dx": torch.empty_like(dy), "dweight": torch.empty_like(weight), "dbias": torch.empty_like(weight), "dresidual": torch.empty_like(dy)}
        LN.layer_norm_backward(ctx, dy, got["sum"], got["mean"], got["rstd"], weight=weight, dropout=drop, work=LN.workspace(ctx, rows, cols), **g)
        check_all(dtype, wtype, g, NU.backward(f64(dy), f64(got["sum"]), f64(got["mean"]), f64(got["rstd"]), f64(weight), None, spec(drop)))


@pytest.mark.parametrize("cols", [96, 700, 4096, 17000])
def test_gradient_against_differences(ctx, cols):
    """fp32: the loss sum(c out) by differences of the kernel's own formula in 64 bits."""
    rows, h = 3, 1e-4
    x, res, c = make(rows, cols, "f32", 0, 1), make(rows, cols, "f32", 0, 2), make(rows, cols, "f32", 0, 3)
    weight, bias, drop = vector(cols, "f32", 4, 0.2, 1.0), vector(cols, "f32", 5), AD.Dropout(0.3, 11)
    f = run_forward(ctx, x, res, weight, bias, 1e-5, drop)
    g = {k: torch.empty_like(t) for k, t in (("dx", x), ("dresidual", x), ("dweight", weight), ("dbias", bias))}
    LN.layer_norm_backward(ctx, c, f["sum"], f["mean"], f["rstd"], weight=weight, dropout=drop, work=LN.workspace(ctx, rows, cols), **g)

    def loss(**change):
        v = {"x": f64(x), "res": f64(res), "weight": f64(weight), "bias": f64(bias)}
        for k, d in change.items():
            v[k] = v[k] + d
        return (f64(c) * NU.forward(v["x"], v["res"], v["weight"], v["bias"], 1e-5, spec(drop))["out"][0]).sum()

    rng = np.random.default_rng(1)
    for arg, grad in (("x", "dx"), ("res", "dresidual"), ("weight", "dweight"), ("bias", "dbias")):
        d = rng.standard_normal(f64(g[grad]).shape)
        slope = (loss(**{arg: h * d}) - loss(**{arg: -h * d})) / (2 * h)
        # (the difference's own error is h^2 of third derivatives; the kernel's 32 bits)
        assert abs(slope - (f64(g[grad]) * d).sum()) <= 1e-4 * np.abs(f64(g[grad]) * d).sum() ** 0.5 * max(1.0, abs(slope)) ** 0.5 + 1e-4


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 0.5, 0.999, 1.0])
def test_probabilities(ctx, dtype, p):
    """Masks that keep everything, little and nothing, on rows with and without whole vectors."""
    for cols in (100, 1024, 777, 17000):
        x, res, dy = make(9, cols, dtype, 0, 1), make(9, cols, dtype, 0, 2), make(9, cols, dtype, 0, 3)
        drop = AD.Dropout(p, 5, 1 << 33)
        got = run_forward(ctx, x, res, None, None, 1e-5, drop)
        check_all(dtype, dtype, got, NU.forward(f64(x), f64(res), None, None, 1e-5, spec(drop)))
        g = {"dx": torch.empty_like(x), "dresidual": torch.empty_like(x)}
        LN.layer_norm_backward(ctx, dy, got["sum"], got["mean"], got["rstd"], dropout=drop, work=LN.workspace(ctx, 9, cols), **g)
        check_all(dtype, dtype, g, NU.backward(f64(dy), f64(got["sum"]), f64(got["mean"]), f64(got["rstd"]), None, None, spec(drop)))
        if p == 1.0:
            assert (g["dx"] == 0).all() and torch.equal(got["sum"], res)
        if p < 2.0 ** -17:
            assert torch.equal(g["dx"], g["dresidual"])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [256, 768, 2048, 4096, 8192, 16384, 20000])
def test_strides_and_alignment_change_nothing(ctx, dtype, cols):
    """Rows apart, rows and weights off 16 bytes: the same results, to the last bit, as whole
    vectors side by side."""
    rows = 21
    src = [make(rows, cols, dtype, 0, i) for i in range(4)]
    weight, bias, drop = vector(cols, "f32", 5, 0.2, 1.0), vector(cols, "f32", 6), AD.Dropout(0.3, 2)
    work, results = LN.workspace(ctx, rows, cols), []
    for off, extra, weights_off in ((0, 0, 0), (16, 64, 0), (3, 6, 0), (0, 0, 1), (5, 7, 3)):
        def place(t):
            wide = torch.zeros(rows, cols + extra, dtype=t.dtype, device="cuda")
            wide[:, off:off + cols] = t
            return wide[:, off:off + cols]

        def shifted(t):
            flat = torch.zeros(cols + weights_off, device="cuda")
            flat[weights_off:] = t
            return flat[weights_off:]

        x, res, dy, dsum = (place(t) for t in src)
        w, b = shifted(weight), shifted(bias)
        f = {"out": place(src[0]), "sum": place(src[0]), "mean": torch.empty(rows, device="cuda"), "rstd": torch.empty(rows, device="cuda")}
        LN.layer_norm(ctx, x, f["out"], weight=w, bias=b, residual=res, dropout=drop, sum=f["sum"], mean=f["mean"], rstd=f["rstd"])
        g = {"dx": place(src[0]), "dresidual": place(src[0]), "dweight": torch.empty(cols, device="cuda"), "dbias": torch.empty(cols, device="cuda")}
        LN.layer_norm_backward(ctx, dy, f["sum"], f["mean"], f["rstd"], weight=w, dsum=dsum, dropout=drop, work=work, **g)
        results.append({**f, **g})
    for r in results[1:]:
        assert all(torch.equal(r[k], results[0][k]) for k in r)


def test_in_place_and_neighbours(ctx):
    for dtype in DT:
        for cols in (96, 100, 1024, 18000):
            x, res = make(40, cols, dtype, 0, 1), make(40, cols, dtype, 0, 2)
            weight, bias, drop = vector(cols, dtype, 3), vector(cols, dtype, 4), AD.Dropout(0.4, 5)
            want = run_forward(ctx, x, res, weight, bias, 1e-5, drop)
            for out_is, sum_is in (("x", "res"), ("res", "x"), (None, "res"), ("x", None)):
                a = {"x": x.clone(), "res": res.clone()}
                out, total = a.get(out_is, torch.empty_like(x)), a.get(sum_is, torch.empty_like(x))
                LN.layer_norm(ctx, a["x"], out, weight=weight, bias=bias, residual=a["res"], dropout=drop, sum=total)
                assert torch.equal(out, want["out"]) and torch.equal(total, want["sum"])
            wide = torch.full((40, cols + 64), 3.0, dtype=DT[dtype], device="cuda")
            LN.layer_norm(ctx, x, wide[:, 9:9 + cols], weight=weight, bias=bias, residual=res, dropout=drop)
            assert torch.equal(wide[:, 9:9 + cols], want["out"])
            assert (wide[:, :9] == 3).all() and (wide[:, 9 + cols:] == 3).all()
            # the gradient: outputs in the place of inputs
            dy, dsum, work = make(40, cols, dtype, 0, 6), make(40, cols, dtype, 0, 7), LN.workspace(ctx, 40, cols)
            g = {k: torch.empty_like(t) for k, t in (("dx", dy), ("dresidual", dy), ("dweight", weight), ("dbias", weight))}
            LN.layer_norm_backward(ctx, dy, want["sum"], want["mean"], want["rstd"], weight=weight, dsum=dsum, dropout=drop, work=work, **g)
            for p, q in (("dy", "sum"), ("sum", "dsum"), ("dsum", "dy"), ("dy", None), (None, "dsum")):
                a = {"dy": dy.clone(), "sum": want["sum"].clone(), "dsum": dsum.clone()}
                dx, dres = a.get(p, torch.empty_like(dy)), a.get(q, torch.empty_like(dy))
                dw, db = torch.empty_like(weight), torch.empty_like(weight)
                LN.layer_norm_backward(ctx, a["dy"], a["sum"], want["mean"], want["rstd"], weight=weight, dsum=a["dsum"], dropout=drop,
                                       dx=dx, dresidual=dres, dweight=dw, dbias=db, work=work)
                assert torch.equal(dx, g["dx"]) and torch.equal(dres, g["dresidual"]) and torch.equal(dw, g["dweight"]) and torch.equal(db, g["dbias"])


def test_is_dropout_then_norm(ctx):
    """The sum is what `dropout` gives, bit for bit."""
    for dtype in DT:
        for cols in (64, 333, 4096):
            x, res, drop = make(50, cols, dtype, 0, 1), make(50, cols, dtype, 0, 2), AD.Dropout(0.3, 9, 77)
            want = torch.empty_like(x)
            AD.dropout(ctx, x, want, drop, residual=res)
            assert torch.equal(run_forward(ctx, x, res, None, None, 1e-5, drop)["sum"], want)


def test_rows_by_themselves(ctx):
    """A row's result does not depend on the others: rows one by one, with the mask's
    offset moved on, and one row for all by a stride of 0."""
    for dtype in DT:
        for cols in (40, 1000, 5000):
            x, res, drop = make(23, cols, dtype, 0, 1), make(23, cols, dtype, 0, 2), AD.Dropout(0.25, 5, 11)
            weight, bias = vector(cols, dtype, 3), vector(cols, dtype, 4)
            want = run_forward(ctx, x, res, weight, bias, 1e-5, drop)
            for t in (0, 7, 22):
                got = run_forward(ctx, x[t:t + 1], res[t:t + 1], weight, bias, 1e-5, drop.advance(t, cols))
                assert all(torch.equal(got[k], want[k][t:t + 1]) for k in want)
            same = run_forward(ctx, x[:1].expand(23, cols), None, weight, bias, 1e-5, None)
            one = run_forward(ctx, x[:1], None, weight, bias, 1e-5, None)
            assert all(torch.equal(same[k], one[k].expand_as(same[k])) for k in same)


def test_infinities_and_nans_stay_in_their_rows(ctx):
    for dtype in DT:
        for cols in (64, 1000, 4096, 17000):
            x = make(12, cols, dtype, 0, 1)
            clean = run_forward(ctx, x, None, None, None, 1e-5, None)
            x[3, cols // 2], x[5, 0], x[7, cols - 1] = float("inf"), float("nan"), float("-inf")
            got = run_forward(ctx, x, None, None, None, 1e-5, None)
            bad = [3, 5, 7]
            good = [t for t in range(12) if t not in bad]
            assert torch.isnan(got["out"][bad]).all() and torch.isnan(got["rstd"][bad]).all()
            assert all(torch.equal(got[k][good], clean[k][good]) for k in got)
            # what is dropped does not count, whatever it held
            drop = AD.Dropout(0.5, 3)
            keep = torch.from_numpy(keep_mask(12, cols, 0.5, 3, 0)).cuda()
            y = torch.where(keep, make(12, cols, dtype, 0, 2), float("nan"))
            z = torch.where(keep, y, 0.0)
            a, b = run_forward(ctx, y, None, None, None, 1e-5, drop), run_forward(ctx, z, None, None, None, 1e-5, drop)
            assert all(torch.equal(a[k], b[k]) for k in a)


def test_flat_rows_and_far_means(ctx):
    """Rows of one value: out = bias, rstd = 1 / sqrt(eps).  A mean that is large beside the
    spread: within what norm_util allows, far below the rounding of the mean in fp32."""
    for cols in (1, 3, 256, 1000, 4096, 20000):
        x = torch.full((5, cols), 1000.3, device="cuda")
        bias = vector(cols, "f32", 1)
        got = run_forward(ctx, x, None, None, bias, 1e-5, None)
        check_all("f32", "f32", got, NU.forward(f64(x), None, None, f64(bias), 1e-5))
        assert (got["rstd"] - 1e5 ** 0.5).abs().max() < 0.01
        if cols > 3:
            x = make(5, cols, "f32", 0, 2, 1.0, 3e4)
            got = run_forward(ctx, x, None, None, None, 1e-5, None)
            check_all("f32", "f32", got, NU.forward(f64(x), None, None, None, 1e-5))
            assert (got["out"].double().mean(1).abs() < 2e-6 * cols ** 0.5 + 1e-5).all()


def test_no_rows(ctx):
    for dtype in DT:
        x = make(0, 64, dtype)
        weight = vector(64, dtype, 1)
        got = run_forward(ctx, x, None, weight, None, 1e-5, None)
        dw, db = torch.full_like(weight, 7), torch.full_like(weight, 7)
        LN.layer_norm_backward(ctx, x, x, got["mean"], got["rstd"], weight=weight, dweight=dw, dbias=db)
        assert (dw == 0).all() and (db == 0).all()


def test_many_rows(ctx):
    """Element offsets past 32 bits; a long sum over the rows."""
    rows, cols = 4_500_000, 1000
    row = make(1, cols, "f16", 0, 1)
    x = row.expand(rows, cols)
    out, mean, rstd = torch.empty(rows, cols, dtype=torch.float16, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    drop = AD.Dropout(0.5, 21)
    LN.layer_norm(ctx, x, out, dropout=drop, mean=mean, rstd=rstd)
    tail = run_forward(ctx, x[:50], None, None, None, 1e-5, drop.advance(rows - 50, cols))
    assert torch.equal(out[-50:], tail["out"]) and torch.equal(mean[-50:], tail["mean"])
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    LN.layer_norm_backward(ctx, out, x, mean, rstd, dx=out, dropout=drop, dweight=dw, dbias=db, work=LN.workspace(ctx, rows, cols))
    back = {"dx": torch.empty(50, cols, dtype=torch.float16, device="cuda")}
    LN.layer_norm_backward(ctx, tail["out"], x[:50], mean[-50:], rstd[-50:], dropout=drop.advance(rows - 50, cols),
                           work=LN.workspace(ctx, 50, cols), **back)
    assert torch.equal(out[-50:], back["dx"])
    ones = torch.ones(1, cols, dtype=torch.float16, device="cuda").expand(rows, cols)
    mean.zero_()
    rstd.fill_(1.0)
    LN.layer_norm_backward(ctx, ones, x, mean, rstd, dweight=dw, dbias=db, work=LN.workspace(ctx, rows, cols))
    c = NU.column_chain_of(rows) * 2.0 ** -24
    assert (db.double() / rows - 1).abs().max() <= c
    assert (dw.double() / rows - row[0].double()).abs().max() <= (c + 2.0 ** -22) * float(row.abs().max())


def test_sums_of_a_billion_rows(ctx):
    """A thread's sums of 512 rows of 1 + 2^-14, and those of a block, are exact; how many blocks'
    sums are added up after that does not show: 40 additions at most are rounded at their own size."""
    rows = 1 << 30
    dy = torch.full((1, 1), 1 + 2.0 ** -14, device="cuda").expand(rows, 1)
    zero, one = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    dw, db = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    LN.layer_norm_backward(ctx, dy, dy, zero, one, dweight=dw, dbias=db, work=LN.workspace(ctx, rows, 1))
    assert abs(float(db) / rows / (1 + 2.0 ** -14) - 1) <= 40 * 2.0 ** -24


def test_squares_of_a_million_columns(ctx):
    """Equal squares, whose additions all round one way: at most 64 + 32 + 21 one after another
    (a rounding of the sum is half of one of rstd), and eight roundings of rstd itself."""
    cols, v = 1 << 20, 1.984375
    x = torch.full((2, cols), v, device="cuda")
    x[:, ::2] = -v
    out, rstd = torch.empty_like(x), torch.empty(2, device="cuda")
    LN.layer_norm(ctx, x, out, rstd=rstd)
    assert (rstd.double() * (v * v + 1e-5) ** 0.5 - 1).abs().max() <= (117 / 2 + 8) * 2.0 ** -24


def test_streams_and_graphs(ctx):
    """Calls on another stream; a captured forward and backward pass, replayed on new
    inputs, beside the eager calls."""
    x, res, dy = make(200, 768, "bf16", 0, 1), make(200, 768, "bf16", 0, 2), make(200, 768, "bf16", 0, 3)
    weight, bias, drop = vector(768, "f32", 4, 0.2, 1.0), vector(768, "f32", 5), AD.Dropout(0.1, 3)
    work = LN.workspace(ctx, 200, 768)

    def call(stream, work):
        f = run_forward(ctx, x, res, weight, bias, 1e-5, drop, stream=stream)
        g = {"dx": torch.empty_like(dy), "dresidual": torch.empty_like(dy), "dweight": torch.empty_like(weight), "dbias": torch.empty_like(bias)}
        LN.layer_norm_backward(ctx, dy, f["sum"], f["mean"], f["rstd"], weight=weight, dropout=drop, work=work, stream=stream, **g)
        return list(f.values()) + list(g.values())

    want = [t.clone() for t in call(None, work)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call(s, work)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call(torch.cuda.current_stream(), work)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, held))
    x.copy_(make(200, 768, "bf16", 0, 9))
    dy.copy_(make(200, 768, "bf16", 0, 10))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    new = call(None, LN.workspace(ctx, 200, 768))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(new, held))
    assert not torch.equal(new[0], want[0])


FIRST_CALLS = """
import sys
sys.path[:0] = [%r]
import torch
from paper_2609_35352_gb300 import adapters as AD, fiona as F, layernorm as LN, optim as O, workloads as W
ctx = F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)
x, w = torch.randn(300, 4096, device="cuda").bfloat16(), torch.ones(4096, device="cuda")
out, total, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
mean, rstd, work = torch.empty(300, device="cuda"), torch.empty(300, device="cuda"), LN.workspace(ctx, 300, 4096)
p, g = torch.randn(2000000, device="cuda").bfloat16(), torch.randn(2000000, device="cuda").bfloat16()
opts = [O.AdamW(ctx, [p.clone()], [g], state_bits=b, max_norm=1.0) for b in (8, 32)]
torch.cuda.synchronize()
def calls():
    s = torch.cuda.current_stream()
    LN.layer_norm(ctx, x, out, weight=w, dropout=AD.Dropout(0.1, 1), sum=total, mean=mean, rstd=rstd, stream=s)
    LN.layer_norm_backward(ctx, x, total, mean, rstd, weight=w, dx=dx, dweight=dw, work=work, stream=s)
    for o in opts:
        o.step(stream=s)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (out, dx, dw)]
assert [o.steps.tolist() for o in opts] == [[1], [1]]
calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (out, dx, dw)))
print("well")
"""


def test_first_calls_in_a_capture(ctx):
    """A program whose very first calls are captured ones."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % root], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "well" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 3, 8, 776, 777, 5003, 20000, 20001])
def test_gradient_of_flat_rows_far_from_zero(ctx, dtype, cols):
    """Rows of one value: xh is 0 at every column, whatever (0 - mean) rstd would be behind the last."""
    dy, s, dsum = make(9, cols, dtype, 0, 1), make(9, cols, dtype, 0, 2, 2.0, 0.5), make(9, cols, dtype, 0, 3)
    mean, rstd = s.double().mean(1).float(), (s.double().var(1, unbiased=False) + 1e-5).rsqrt().float()
    weight, work = vector(cols, dtype, 4, 0.2, 1.0), LN.workspace(ctx, 9, cols)

    def call(extra):
        g = {"dx": torch.empty_like(dy), "dresidual": torch.empty_like(dy), "dweight": torch.empty_like(weight), "dbias": torch.empty_like(weight)}
        LN.layer_norm_backward(ctx, dy, s, mean, rstd, weight=weight, dsum=extra, work=work, **g)
        return g

    clean = [call(extra) for extra in (None, dsum)]
    flat = {2: 2e36, 5: torch.finfo(DT[dtype]).min, 7: 1e33}
    for t, value in flat.items():
        s[t] = value
        mean[t], rstd[t] = s[t, 0].float(), 1e-5 ** -0.5 if t != 7 else 1e-12 ** -0.5
    good = [t for t in range(9) if t not in flat]
    for extra, before in zip((None, dsum), clean):
        got = call(extra)
        check_all(dtype, dtype, got, NU.backward(f64(dy), f64(s), f64(mean), f64(rstd), f64(weight), f64(extra)))
        assert all(torch.equal(got[k][good], before[k][good]) for k in ("dx", "dresidual"))


@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("cols", [1, 3, 8, 100, 512, 777, 1024, 2048, 4096, 5000, 8192, 16384, 17000, 20001])
def test_finite_rows_past_the_range_of_sums(ctx, dtype, wtype, cols):
    """Rows of finite values whose sum, squares or distances from the mean pass fp32's range come
    out by the formula (the bound of its rounding is that of any row), others as without them."""
    weight, bias = vector(cols, wtype, 3, 0.2, 1.0), vector(cols, wtype, 4)
    for drop, res, scale in ((None, None, 1.0), (AD.Dropout(0.5, 9), make(12, cols, dtype, 0, 2), 0.25)):
        x = make(12, cols, dtype, 0, 1)
        clean = run_forward(ctx, x, res, weight, bias, 1e-5, drop)
        signs = torch.where(torch.arange(cols, device="cuda") % 2 == 0, 1.0, -1.0)
        first = torch.where(torch.arange(cols, device="cuda") == 0, -1.0, 1.0)
        noise = make(1, cols, "f32", 0, 5)[0]
        far = {1: torch.full((cols,), 1e38, device="cuda"), 2: noise * 3e37, 4: signs * 3.3e38, 5: first * 3.3e38, 6: noise * 1e25,
               8: noise * 1e18, 9: torch.full((cols,), torch.finfo(DT[dtype]).min, device="cuda"), 11: noise * 1e37 - 1e38}
        for t, row in far.items():
            x[t] = (row * scale).to(DT[dtype])
        assert torch.isfinite(x).all()
        got = run_forward(ctx, x, res, weight, bias, 1e-5, drop)
        check_all(dtype, wtype, got, NU.forward(f64(x), f64(res), f64(weight), f64(bias), 1e-5, spec(drop)))
        good = [t for t in range(12) if t not in far]
        assert all(torch.equal(got[k][good], clean[k][good]) for k in got)
        plain = torch.empty_like(x)
        LN.layer_norm(ctx, x, plain, weight=weight, bias=bias, residual=res, dropout=drop)
        assert torch.equal(plain, got["out"])
        # alone, and with rows of an infinity or a NaN beside them
        for t in (2, 4, 6):
            d = None if drop is None else drop.advance(t, cols)
            one = run_forward(ctx, x[t:t + 1], None if res is None else res[t:t + 1], weight, bias, 1e-5, d)
            assert all(torch.equal(one[k], got[k][t:t + 1]) for k in got)
        if drop is None:
            x[0, cols - 1], x[3, 0] = float("inf"), float("nan")
            bad = run_forward(ctx, x, None, weight, bias, 1e-5, None)
            assert torch.isnan(bad["out"][[0, 3]]).all() and torch.isnan(bad["rstd"][[0, 3]]).all()
            rest = [t for t in range(12) if t not in (0, 3)]
            assert all(torch.equal(bad[k][rest], got[k][rest]) for k in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [64, 256, 512, 768, 1024, 2048, 4096, 8192, 16384, 20000])
def test_far_rows_by_any_path(ctx, dtype, cols):
    """Rows past the range of sums: to the last bit the same off 16 bytes and in place of the inputs."""
    src, res = make(7, cols, dtype, 0, 1), make(7, cols, dtype, 0, 2)
    src[1], src[2], src[4] = (src[1].float() * 3e37).to(DT[dtype]), (src[2].float() * 1e25).to(DT[dtype]), 1e38
    src[5, 1::2] = -3e38
    weight, bias, drop = vector(cols, "f32", 3, 0.2, 1.0), vector(cols, "f32", 4), AD.Dropout(0.25, 3)
    results = []
    for off in (0, 1, 8):
        def place(t):
            wide = torch.zeros(7, cols + 2 * off, dtype=t.dtype, device="cuda")
            wide[:, off:off + cols] = t
            return wide[:, off:off + cols]

        for in_place in (False, True):
            x, r = place(src), place(res)
            out, total = (r, x) if in_place else (place(src), place(src))
            mean, rstd = torch.empty(7, device="cuda"), torch.empty(7, device="cuda")
            LN.layer_norm(ctx, x, out, weight=weight, bias=bias, residual=r, dropout=drop, sum=total, mean=mean, rstd=rstd)
            results.append((out, total, mean, rstd))
    finite = torch.isfinite(results[0][1]).all(1)  # (what is kept grows by the dropout's factor)
    assert finite.sum() >= 6 and torch.isfinite(results[0][0][finite]).all() and torch.isfinite(results[0][3][finite]).all()
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip((t[finite] for t in r), (t[finite] for t in results[0])))
