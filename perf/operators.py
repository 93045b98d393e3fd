"""Performance cases of the low-rank adapters beside a shared projection and of
the dropout whose mask is never stored: what a program that serves or trains
them does, from one token of one client to a training batch.

A case is one pass of one of five operations:

  forward           out = base + s_a (x A_a^T) B_a^T over the rows of every
                    request, `base` being the shared projection's output:
                    serving, from single tokens to prompts
  train             the same of D(x), D a dropout, returning h = D(x) A_a^T
                    for the gradient too
  backward          dx, dA and dB of `train`, from x, h and dy
  dropout           residual + D(x)
  dropout_backward  D'(dy), the same mask

D keeps element (t, i) of [rows, cols] where the 16-bit field i % 4 of value
number offset + t ceil(cols / 4) + i / 4 of a SplitMix64 stream is at least
65536 p, and divides by 1 - p (p rounded to a multiple of 2^-16); the stream's
key is its value number 4 under the seed.

The context, the batch of requests (who owns which rows, and the adapters'
ranks and scales) and the adapters' weights are what such a program keeps
between calls, its workspace and output buffers too.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
DROPOUT_STREAM = 4


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------
def _adapters(op, dtype, tokens, requests, adapters, rank, d_in, d_out, mixed=False, p=0.0, name=None):
    c = {"op": op, "dtype": dtype, "tokens": tokens, "requests": requests, "adapters": adapters, "rank": rank,
         "d_in": d_in, "d_out": d_out, "mixed": mixed, "p": p}
    return dict(c, name=name) if name else c


def _dropout(op, dtype, rows, cols, p, name=None):
    c = {"op": op, "dtype": dtype, "rows": rows, "cols": cols, "p": p}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one client beside a 768 -> 768 projection: all latency
        _adapters("forward", "bf16", 1, 1, 1, 8, 768, 768, name="serve-one"),
        # a step of 64 clients, most with their own adapter
        _adapters("forward", "bf16", 64, 64, 48, 16, 4096, 4096, name="serve-64"),
        # a step of many clients beside a wide projection, ranks from 16 to 64
        _adapters("forward", "f16", 256, 256, 200, 64, 2048, 8192, mixed=True, name="serve-256-wide"),
        # prompts of 24 clients at once, ranks from 8 to 32, one without an adapter
        _adapters("forward", "bf16", 8192, 24, 8, 32, 4096, 4096, mixed=True, name="prompts"),
        # activations as they come out of decryption, in 32 bits
        _adapters("forward", "f32", 2048, 6, 4, 16, 1024, 1024, name="prompts-f32"),
        # no size a multiple of anything
        _adapters("forward", "f16", 1531, 9, 5, 13, 1001, 777, mixed=True, name="prompts-odd"),
        # fine-tuning one client's adapter on a long batch
        _adapters("train", "bf16", 16384, 1, 1, 32, 4096, 4096, p=0.05, name="train"),
        _adapters("backward", "bf16", 16384, 1, 1, 32, 4096, 4096, p=0.05, name="train-backward"),
        # a small batch of four clients in 32 bits
        _adapters("backward", "f32", 2048, 4, 4, 8, 768, 768, p=0.1, name="train-backward-f32"),
        # two clients, a high rank, a wide projection
        _adapters("backward", "f16", 4096, 2, 2, 128, 2048, 8192, name="train-backward-wide"),
        # the dropout of a block's output on its way into the residual stream
        _dropout("dropout", "bf16", 16384, 4096, 0.1, name="dropout-residual"),
        # the gradient through it, odd sizes
        _dropout("dropout_backward", "f32", 1531, 777, 0.1, name="dropout-backward-odd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    step = rng.choice([1, 8, 64, 64])
    return max(lo, n // step * step)


def draw(rng):
    op = rng.choice(["forward", "forward", "forward", "train", "backward", "backward", "dropout", "dropout_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("dropout"):
        c = _dropout(op, dtype, _log(rng, 16, 16384), _width(rng, 64, 8192), rng.choice([0.05, 0.1, 0.2, 0.5]))
        rows = "rows"
    else:
        tokens = _log(rng, 1, 16384)
        single = op == "forward" and tokens <= 512 and rng.random() < 0.7
        requests = tokens if single else min(tokens, _log(rng, 1, 32))
        rank = rng.choice([8, 16, 32, 64, 128, rng.randint(2, 64)])
        c = _adapters(op, dtype, tokens, requests, _log(rng, 1, max(1, min(requests, 256))), rank,
                      _width(rng, 64, 8192), _width(rng, 64, 8192), mixed=rng.random() < 0.5,
                      p=0.0 if op == "forward" else rng.choice([0.0, 0.05, 0.1]))
        rows = "tokens"
    top = [work(t) for t in listed()]
    most = {k: max(t[k] for t in top) for k in ("bytes", "flops")}
    while any(work(c)[k] > most[k] for k in most):
        c[rows] = c[rows] * 3 // 4
        if rows == "tokens":
            c["requests"] = min(c["requests"], c["tokens"])
            c["adapters"] = min(c["adapters"], c["requests"])
    return c


def _composition(c):
    """starts[requests + 1], the adapter of each request and each adapter's rank.
    Requests of one token each, or of uneven lengths, an empty one among them."""
    rng = random.Random("%(tokens)d %(requests)d %(adapters)d" % c)
    n, T = c["requests"], c["tokens"]
    if n == T:
        lengths = [1] * n
    else:
        share = [rng.uniform(0.5, 1.5) for _ in range(n)]
        if n >= 6:
            share[3] = 0.0
        cut = [0] + [round(T * sum(share[:i + 1]) / sum(share)) for i in range(n)]
        lengths = [cut[i + 1] - cut[i] for i in range(n)]
    starts = [0]
    starts += [sum(lengths[:i + 1]) for i in range(n)]
    ids = [i % c["adapters"] for i in range(n)]
    rng.shuffle(ids)
    if n >= 6 and n != T:
        ids[2] = -1
    ranks = [max(1, c["rank"] >> (i % 3)) if c["mixed"] else c["rank"] for i in range(c["adapters"])]
    return starts, ids, ranks


def work(c):
    e = SIZE[c["dtype"]]
    if c["op"].startswith("dropout"):
        n = c["rows"] * c["cols"]
        return {"bytes": (3 if c["op"] == "dropout" else 2) * n * e, "flops": 2 * n}
    starts, ids, ranks = _composition(c)
    d = c["d_in"] + c["d_out"]
    rows = [b - a for a, b in zip(starts, starts[1:])]
    used = {a for a, n in zip(ids, rows) if a >= 0 and n}
    live = sum(n for a, n in zip(ids, rows) if a >= 0)
    weights = sum(ranks[a] for a in used) * d * e
    products = sum(n * ranks[a] for a, n in zip(ids, rows) if a >= 0) * d
    T = c["tokens"]
    if c["op"] == "backward":
        grads = c["adapters"] * c["rank"] * d * e
        return {"bytes": (live * d + T * c["d_in"]) * e + 4 * live * c["rank"] + weights + grads, "flops": 4 * products}
    saved = 4 * T * c["rank"] if c["op"] == "train" else 0
    return {"bytes": (live * c["d_in"] + 2 * T * c["d_out"]) * e + weights + saved, "flops": 2 * products}


# ----------------------------------------------------------------------------
# what a program has before the call
# ----------------------------------------------------------------------------
def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)

    s = {"rng_seed": (seed * 0x9E3779B1 + 12345) % (1 << 63), "rng_offset": (seed % 1000) * 1000003}
    if c["op"].startswith("dropout"):
        s["x"] = normal(c["rows"], c["cols"])
        if c["op"] == "dropout":
            s["residual"] = normal(c["rows"], c["cols"], scale=3.0)
        return s
    T, r = c["tokens"], c["rank"]
    s["x"] = normal(T, c["d_in"])
    s["A"] = normal(c["adapters"], r, c["d_in"], scale=c["d_in"] ** -0.5)
    s["B"] = normal(c["adapters"], c["d_out"], r, scale=0.5 * r ** -0.5)
    s["scales"] = [2.0 / (1 + a % 3) for a in range(c["adapters"])]
    if c["op"] == "backward":
        s["dy"] = normal(T, c["d_out"], scale=0.1)
    else:
        s["base"] = normal(T, c["d_out"])
    return s


_context = None


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    dt, dev = DTYPES[case["dtype"]], "cuda"
    if case["op"].startswith("dropout"):
        s["out"] = torch.empty_like(s["x"])
    else:
        starts, ids, ranks = _composition(case)
        T, R = case["tokens"], case["requests"]
        lengths = [b - a for a, b in zip(starts, starts[1:])]
        most = max(lengths)
        owner = np.repeat(np.arange(R), lengths)
        within = np.arange(T) - np.asarray(starts)[owner]
        rows = np.minimum(np.asarray(starts[:-1])[:, None] + np.arange(most), T - 1)
        inside = np.arange(most) < np.asarray(lengths)[:, None]
        rank = np.asarray([ranks[a] if a >= 0 else 0 for a in ids])
        s["starts"], s["ids"], s["ranks"] = starts, ids, ranks
        # the same for the plain form: each request's rows, padded to the longest
        s["rows"] = torch.from_numpy(rows).to(dev)
        s["at"] = torch.from_numpy(owner * most + within).to(dev)
        s["inside"] = torch.from_numpy(inside).to(dev)[:, :, None]
        s["adapter"] = torch.tensor([max(a, 0) for a in ids], device=dev)
        s["live"] = torch.from_numpy(np.arange(case["rank"]) < rank[:, None]).to(dev)[:, None, :]
        s["scale"] = torch.tensor([s["scales"][max(a, 0)] for a in ids], device=dev)[:, None, None]
        s["of"] = torch.tensor([[float(a == j) for a in ids] for j in range(case["adapters"])], device=dev)
        if case["op"] == "backward":
            s["h"] = _plain_h(s)
            s["dx"], s["dA"], s["dB"] = torch.empty_like(s["x"]), torch.empty_like(s["A"]), torch.empty_like(s["B"])
        else:
            s["out"] = torch.empty_like(s["base"])
            s["h"] = torch.empty(T, case["rank"], device=dev) if case["op"] == "train" else None
    if own:
        from paper_2609_35352_gb300 import adapters, fiona, workloads
        global _context
        if _context is None:
            _context = fiona.Context(1024, workloads.ntt_primes(1024, 50, 1), device=0)
        s["ctx"] = _context
        s["drop"] = adapters.Dropout(case["p"], s["rng_seed"], s["rng_offset"]) if case["p"] else None
        if not case["op"].startswith("dropout"):
            s["batch"] = adapters.Batch(_context, s["starts"], s["ids"], s["ranks"], case["rank"], s["scales"])
            s["work"] = s["batch"].workspace(case["d_in"], case["d_out"], dt)
    return s


# ----------------------------------------------------------------------------
# the plain form
# ----------------------------------------------------------------------------
def _mul64(z, by):
    return z * (by - (1 << 64) if by >> 63 else by)  # (int64 products wrap)


def _xor_shift(z, n):
    return z ^ ((z >> n) & ((1 << (64 - n)) - 1))


def _mix(z):
    m = (1 << 64) - 1
    z = ((z ^ (z >> 30)) * MIX1) & m
    z = ((z ^ (z >> 27)) * MIX2) & m
    return z ^ (z >> 31)


def _key(seed):
    return _mix((seed + (DROPOUT_STREAM + 1) * GOLDEN) & ((1 << 64) - 1))


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _plain_dropout(x, s):
    """D(x) in 32 bits: dropped elements are zero, whatever they held."""
    rows, cols = x.shape
    groups = (cols + 3) // 4
    n = torch.arange(rows * groups, device=x.device).view(rows, groups)
    z = _mul64(n, GOLDEN) + _signed(_key(s["rng_seed"]) + (s["rng_offset"] + 1) * GOLDEN)
    z = _mul64(_xor_shift(z, 30), MIX1)
    z = _mul64(_xor_shift(z, 27), MIX2)
    z = _xor_shift(z, 31)
    fields = (z[:, :, None] >> torch.arange(0, 64, 16, device=x.device)) & 0xFFFF
    level = round(s["case"]["p"] * 65536)
    keep = fields.view(rows, 4 * groups)[:, :cols] >= level
    return torch.where(keep, x.float() * (65536.0 / (65536 - level)), 0.0)


def _plain_input(s):
    x = _plain_dropout(s["x"], s) if s["case"]["p"] else s["x"].float()
    return torch.where(s["inside"], x[s["rows"]], 0.0)


def _plain_h(s):
    h = torch.bmm(_plain_input(s), s["A"].float()[s["adapter"]].transpose(1, 2))
    return torch.where(s["live"], h, 0.0).flatten(0, 1)[s["at"]]


def _plain_forward(s):
    h = torch.bmm(_plain_input(s), s["A"].float()[s["adapter"]].transpose(1, 2))
    h = torch.where(s["live"], h, 0.0)
    B = torch.where(s["live"], s["B"].float()[s["adapter"]], 0.0)
    add = s["scale"] * torch.bmm(h, B.transpose(1, 2))
    out = (s["base"].float() + add.flatten(0, 1)[s["at"]]).to(s["base"].dtype)
    return [out, h.flatten(0, 1)[s["at"]]] if s["case"]["op"] == "train" else out


def _plain_backward(s):
    x = _plain_input(s)
    dy = torch.where(s["inside"], s["dy"].float()[s["rows"]], 0.0)
    h = torch.where(s["inside"], s["h"][s["rows"]], 0.0)
    A, B = s["A"].float()[s["adapter"]], s["B"].float()[s["adapter"]]
    dh = torch.where(s["live"], s["scale"] * torch.bmm(dy, B), 0.0)
    dx = torch.bmm(dh, torch.where(s["live"].transpose(1, 2), A, 0.0)).flatten(0, 1)[s["at"]]
    if s["case"]["p"]:
        dx = _plain_dropout(dx, s)
    dA = torch.bmm(dh.transpose(1, 2), x).flatten(1)
    dB = torch.where(s["live"], s["scale"] * torch.bmm(dy.transpose(1, 2), h), 0.0).flatten(1)
    dt = s["x"].dtype
    return [dx.to(dt), (s["of"] @ dA).view(s["A"].shape).to(dt), (s["of"] @ dB).view(s["B"].shape).to(dt)]


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2609_35352_gb300 import adapters
        stream = torch.cuda.current_stream()
        if op == "dropout":
            adapters.dropout(s["ctx"], s["x"], s["out"], s["drop"], residual=s["residual"], stream=stream)
            return s["out"]
        if op == "dropout_backward":
            adapters.dropout_backward(s["ctx"], s["x"], s["out"], s["drop"], stream=stream)
            return s["out"]
        if op == "backward":
            s["batch"].backward(s["x"], s["h"], s["dy"], s["A"], s["B"], s["dx"], s["dA"], s["dB"], dropout=s["drop"],
                                work=s["work"], stream=stream)
            return [s["dx"], s["dA"], s["dB"]]
        s["batch"].forward(s["x"], s["A"], s["B"], s["out"], base=s["base"], h=s["h"], dropout=s["drop"],
                           work=s["work"], stream=stream)
        return [s["out"], s["h"]] if op == "train" else s["out"]
    if op == "dropout":
        return (s["residual"].float() + _plain_dropout(s["x"], s)).to(s["x"].dtype)
    if op == "dropout_backward":
        return _plain_dropout(s["x"], s).to(s["x"].dtype)
    return _plain_backward(s) if op == "backward" else _plain_forward(s)


# ----------------------------------------------------------------------------
# the definition in 64 bits
# ----------------------------------------------------------------------------
def _exact_keep(rows, cols, p, seed, offset):
    per_row = -(-cols // 4)
    with np.errstate(over="ignore"):
        n = np.arange(1, rows * per_row + 1, dtype=np.uint64) + np.uint64(offset)
        z = np.uint64(_key(seed)) + n * np.uint64(GOLDEN)
        z ^= z >> np.uint64(30)
        z *= np.uint64(MIX1)
        z ^= z >> np.uint64(27)
        z *= np.uint64(MIX2)
        z ^= z >> np.uint64(31)
    return z.astype("<u8").view("<u2").reshape(rows, 4 * per_row)[:, :cols] >= round(p * 65536)


def exact(case, seed):
    v = {k: t.double().cpu().numpy() if torch.is_tensor(t) else t for k, t in _inputs(case, seed).items()}
    x, p = v["x"], case["p"]
    if p:
        keep = _exact_keep(x.shape[0], x.shape[1], p, v["rng_seed"], v["rng_offset"])
        factor = 65536 / (65536 - round(p * 65536))
        x = np.where(keep, x * factor, 0.0)
    if case["op"].startswith("dropout"):
        return x + v["residual"] if case["op"] == "dropout" else x
    starts, ids, ranks = _composition(case)
    A, B = v["A"], v["B"]
    h = np.zeros((case["tokens"], case["rank"]))
    spans = [(slice(b, e), a, ranks[a], v["scales"][a]) for b, e, a in zip(starts, starts[1:], ids) if a >= 0]
    for t, a, k, _ in spans:
        h[t, :k] = x[t] @ A[a, :k].T
    if case["op"] != "backward":
        out = v["base"]
        for t, a, k, scale in spans:
            out[t] += scale * (h[t, :k] @ B[a, :, :k].T)
        return [out, h] if case["op"] == "train" else out
    dy, dx, dA, dB = v["dy"], np.zeros_like(x), np.zeros_like(A), np.zeros_like(B)
    for t, a, k, scale in spans:
        dh = scale * (dy[t] @ B[a, :, :k])
        dx[t] = dh @ A[a, :k]
        dA[a, :k] += dh.T @ x[t]
        dB[a, :, :k] += scale * (dy[t].T @ h[t, :k])
    if p:
        dx = np.where(keep, dx * factor, 0.0)
    return [dx, dA, dB]
