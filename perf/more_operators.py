"""Performance cases of the layer norm with the dropout and the residual before
it, and of the AdamW step over the tensors of many clients at once: what a
program that serves or trains a block in the clear does beside the adapters.

A case is one pass of one of three operations:

  norm           s = residual + D(x), y = gamma (s - mean) rstd + beta by rows;
                 training keeps s, mean and rstd for the gradient, serving of a
                 block whose norm stands before the projection keeps s
  norm_backward  ds = dsum + rstd (g - mean(g) - xh mean(g xh)) with
                 xh = (s - mean) rstd and g = gamma dy; the residual's gradient
                 ds, the input's dx = D'(ds), and the gradients of gamma and
                 beta: sums of dy xh and of dy over the rows
  adamw          one step for every client (a group of tensors' slices with its
                 own step count, learning rate and gradient norm): clipping,
                 moments in 32 or in 8 bits, weights in their own type with or
                 without a 32-bit master copy

D is the dropout of `perf/operators.py`: element (t, i) of [rows, cols] is kept
where the 16-bit field i % 4 of value number offset + t ceil(cols / 4) + i / 4
of a SplitMix64 stream is at least 65536 p, and divided by 1 - p (p rounded to
a multiple of 2^-16); the stream's key is its value number 4 under the seed.

Moments stand in blocks of 256 elements of one slice (the last one filled with
zeros).  In 8 bits a block has one 32-bit scale for m, the largest |m|, and one
for u = sqrt(v), the largest u; m is q |q| / 127^2 of its scale for a q from
-127 to 127, u is q^2 / 255^2 of its scale for a q from 0 to 255 (1 at least
where v > 0), each the nearest such value.  They come back as the values that
they stand for, in bf16 (a code has fewer bits).

The context, the optimizer (its tensors' addresses and its state) and the
output buffers are what such a program keeps between calls.
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
EPS = 1e-5
BLOCK = 256
BETA1, BETA2, ADAM_EPS, DECAY, MAX_NORM = 0.9, 0.999, 1e-8, 0.01, 1.0


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------
def _norm(op, dtype, rows, cols, keep, p=0.0, residual=True, name=None):
    """keep: "all" (s, mean and rstd come back, or dsum goes in), "sum" or "none"."""
    c = {"op": op, "dtype": dtype, "rows": rows, "cols": cols, "keep": keep, "p": p, "residual": residual}
    return dict(c, name=name) if name else c


def _adamw(dtype, clients, layers, rank, d_in, d_out, bits=32, master=False, clip=False, name=None):
    """rank 0: one whole matrix [d_out][d_in] a layer instead of a low-rank pair."""
    c = {"op": "adamw", "dtype": dtype, "clients": clients, "layers": layers, "rank": rank, "d_in": d_in, "d_out": d_out,
         "bits": bits, "master": master, "clip": clip}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the norm after one token's projection, 768 wide: all latency
        _norm("norm", "bf16", 1, 768, "none", name="norm-one"),
        # a serving step of 64 tokens into the residual stream of a wide block
        _norm("norm", "bf16", 64, 4096, "sum", name="norm-64"),
        # a training batch: dropout, residual and norm, with what the gradient needs
        _norm("norm", "bf16", 16384, 4096, "all", p=0.1, name="norm-train"),
        # its gradient
        _norm("norm_backward", "bf16", 16384, 4096, "none", p=0.1, name="norm-train-backward"),
        # activations as they come out of decryption, in 32 bits
        _norm("norm", "f32", 2048, 1024, "none", residual=False, name="norm-f32"),
        # the gradient of wide rows in 32 bits, the residual stream's own gradient coming in
        _norm("norm_backward", "f32", 4096, 8192, "all", name="norm-backward-wide-f32"),
        # no size a multiple of anything
        _norm("norm_backward", "f16", 1531, 777, "none", p=0.1, name="norm-backward-odd"),
        # a step of one client's adapter of one layer: all latency
        _adamw("f32", 1, 1, 8, 768, 768, name="adamw-one"),
        # a step of 64 clients' adapters in 12 layers, each client clipped by its own norm
        _adamw("bf16", 64, 12, 16, 768, 768, master=True, clip=True, name="adamw-clients"),
        # the same of few clients with odd widths, states in 8 bits
        _adamw("f16", 7, 6, 13, 1001, 777, bits=8, clip=True, name="adamw-odd-8bit"),
        # every projection of a model trained whole, 402 million weights
        _adamw("bf16", 1, 24, 0, 4096, 4096, master=True, clip=True, name="adamw-model"),
        # 201 million with states in 8 bits
        _adamw("bf16", 1, 12, 0, 4096, 4096, bits=8, name="adamw-model-8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    step = rng.choice([1, 8, 64, 64])
    return max(lo, n // step * step)


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op != "adamw":
        back = op == "norm_backward"
        c = _norm(op, dtype, _log(rng, 1, 16384), _width(rng, 64, 8192), rng.choice(["all", "none"] if back else ["all", "sum", "none"]),
                  p=rng.choice([0.0, 0.1, 0.2]), residual=back or rng.random() < 0.7)
        key = "rows"
    else:
        whole = rng.random() < 0.3
        c = _adamw(dtype, 1 if whole else _log(rng, 1, 96), _log(rng, 1, 24), 0 if whole else rng.choice([8, 16, 32, 64, rng.randint(2, 64)]),
                   _width(rng, 64, 4096), _width(rng, 64, 4096), bits=rng.choice([32, 32, 8]), master=dtype != "f32" and rng.random() < 0.5,
                   clip=rng.random() < 0.6)
        key = "layers"
    top = [work(t) for t in listed()]
    most = {k: max(t[k] for t in top) for k in ("bytes", "flops")}
    while any(work(c)[k] > most[k] for k in most) and c[key] > 1:
        c[key] = c[key] * 3 // 4
    return c


def _shapes(c):
    """The tensors of an adamw case: [clients][...]."""
    if c["rank"]:
        return [(c["clients"], c["rank"], c["d_in"]), (c["clients"], c["d_out"], c["rank"])] * c["layers"]
    return [(1, c["d_out"], c["d_in"])] * c["layers"]


def _idle(c):
    """A client without data in this step: it stays as it is."""
    return 3 if c["clients"] >= 6 else None


def work(c):
    e = SIZE[c["dtype"]]
    if c["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(c))
        live = n // c["clients"] * (c["clients"] - (_idle(c) is not None))
        state = 4 * 4 if c["bits"] == 32 else 4 + 16 / BLOCK
        per = 2 * e + 8 if c["master"] else 3 * e
        # (8-bit moments come back as values)
        return {"bytes": live * (per + state) + (n * 4 if c["bits"] == 8 else 0), "flops": 16 * live}
    n = c["rows"] * c["cols"]
    if c["op"] == "norm":
        moves = 2 + c["residual"] + (c["keep"] != "none")
        return {"bytes": moves * n * e + (8 * c["rows"] if c["keep"] == "all" else 0) + 2 * c["cols"] * e, "flops": 10 * n}
    moves = 3 + (c["keep"] == "all") + (c["p"] > 0)
    return {"bytes": moves * n * e + 8 * c["rows"] + 3 * c["cols"] * e, "flops": 14 * n}


# ----------------------------------------------------------------------------
# what a program has before the call
# ----------------------------------------------------------------------------
def _norm_inputs(c, g, s):
    dt, rows, cols = DTYPES[c["dtype"]], c["rows"], c["cols"]

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale + shift

    s["weight"] = normal(cols, scale=0.1, shift=1.0).to(dt)
    # a few columns of a residual stream are far larger than the others
    loud = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 12.0, 1.0)
    if c["op"] == "norm":
        s["bias"] = normal(cols, scale=0.1).to(dt)
        s["x"] = (normal(rows, cols) if c["residual"] else normal(rows, cols, scale=2.0, shift=0.5) * loud).to(dt)
        if c["residual"]:
            s["residual"] = (normal(rows, cols, scale=2.0, shift=0.3) * loud).to(dt)
        return
    s["dy"] = normal(rows, cols, scale=0.1).to(dt)
    s["sum"] = (normal(rows, cols, scale=2.0, shift=0.3) * loud).to(dt)
    if c["keep"] == "all":
        s["dsum"] = normal(rows, cols, scale=0.1).to(dt)
    v = s["sum"].double()
    mean = v.mean(1)
    s["mean"], s["rstd"] = mean.float(), (v.var(1, unbiased=False) + EPS).rsqrt().float()


def _adamw_inputs(c, g, s):
    """Everything in flat buffers.  Weights and gradients: the tensors one after
    another, each from a multiple of BLOCK on.  Moments and the master copy: the
    slices one after another, each filled up to whole blocks."""
    dt, shapes, clients = DTYPES[c["dtype"]], _shapes(c), c["clients"]
    slices = np.asarray([math.prod(t[1:]) for t in shapes])
    blocks = -(-slices // BLOCK)
    room = -(-slices * clients // BLOCK) * BLOCK
    s["starts"] = np.concatenate([[0], np.cumsum(room)])
    # each block's client, its first weight and how many it has
    tensor = np.repeat(np.arange(len(shapes)), blocks * clients)
    within = np.arange(len(tensor)) - np.repeat(np.cumsum(blocks * clients) - blocks * clients, blocks * clients)
    client, k = within // blocks[tensor], within % blocks[tensor]
    first = s["starts"][tensor] + client * slices[tensor] + k * BLOCK
    count = np.minimum(BLOCK, slices[tensor] - k * BLOCK)
    s["client"] = torch.from_numpy(client).cuda()
    s["aligned"] = bool((slices % BLOCK == 0).all())
    lane = torch.arange(BLOCK, device="cuda")
    s["inside"] = lane < torch.from_numpy(count).cuda()[:, None]
    if not s["aligned"]:
        s["at"] = torch.where(s["inside"], torch.from_numpy(first).cuda()[:, None] + lane, 0)

    n, nb = int(s["starts"][-1]), len(tensor)
    per_client = int(slices.sum())
    used = torch.ones(n, dtype=torch.bool, device="cuda")
    if not s["aligned"]:
        used.zero_()
        used[s["at"][s["inside"]]] = True
    s["p"] = (torch.randn(n, generator=g, device="cuda") * 0.02 * used).to(dt)
    # gradients of norms from 0.25 to 4: some clients are clipped, others are not
    size = torch.tensor([0.25 * 4 ** (2 * i / max(1, clients - 1)) if clients > 1 else 2.0 for i in range(clients)], device="cuda") * per_client ** -0.5
    gradient = torch.randn(nb, BLOCK, generator=g, device="cuda") * size[s["client"]][:, None]
    if s["aligned"]:
        s["g"] = gradient.view(-1).to(dt)
    else:
        s["g"] = torch.zeros(n, dtype=dt, device="cuda")
        s["g"][s["at"][s["inside"]]] = gradient[s["inside"]].to(dt)
    del gradient
    live = s["inside"] if not s["aligned"] else 1.0
    typical = size[s["client"]][:, None].clamp(max=MAX_NORM * per_client ** -0.5)
    m = torch.randn(nb, BLOCK, generator=g, device="cuda") * (0.3 * typical) * live
    v = (torch.rand(nb, BLOCK, generator=g, device="cuda") + 0.3).square_() * typical ** 2 * live
    if c["bits"] == 8:
        s["m"], s["m_scale"] = _encode_m(m)
        s["v"], s["v_scale"] = _encode_v(v)
    else:
        s["m"], s["v"] = m, v
    if c["master"]:
        w = s["p"].float() if s["aligned"] else torch.where(s["inside"], s["p"][s["at"]].float(), 0.0)
        # (what the weights lost when they were rounded)
        s["master"] = (w.view(nb, BLOCK) * (1 + (torch.rand(nb, BLOCK, generator=g, device="cuda") - 0.5) * torch.finfo(dt).eps))
    s["steps"] = torch.randint(1, 2000, (clients,), generator=g, device="cuda")
    s["lr"] = [1e-3 / (1 + i % 3) for i in range(clients)]
    s["active"] = torch.tensor([i != _idle(c) for i in range(clients)], device="cuda")


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"rng_seed": (seed * 0x9E3779B1 + 12345) % (1 << 63), "rng_offset": (seed % 1000) * 1000003}
    (_adamw_inputs if c["op"] == "adamw" else _norm_inputs)(c, g, s)
    return s


_context = None


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "norm":
        s["out"] = torch.empty_like(s["x"])
        s["sum"] = torch.empty_like(s["x"]) if case["keep"] != "none" else None
        for k in ("mean", "rstd"):
            s[k] = torch.empty(case["rows"], device="cuda") if case["keep"] == "all" else None
    elif case["op"] == "norm_backward":
        s["dx"] = torch.empty_like(s["dy"])
        s["dresidual"] = torch.empty_like(s["dy"]) if case["p"] else None
        s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["weight"])
    else:
        s["rate"] = torch.tensor(s["lr"], device="cuda")
        if case["bits"] == 8:
            s["m_out"], s["v_out"] = (torch.empty(s["m"].shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if own:
        from paper_2609_35352_gb300 import adapters, fiona, layernorm, optim, workloads
        global _context
        if _context is None:
            _context = fiona.Context(1024, workloads.ntt_primes(1024, 50, 1), device=0)
        s["ctx"] = _context
        if case["op"] != "adamw":
            s["drop"] = adapters.Dropout(case["p"], s["rng_seed"], s["rng_offset"]) if case["p"] else None
            if case["op"] == "norm_backward":
                s["work"] = layernorm.workspace(_context, case["rows"], case["cols"])
        else:
            shapes = _shapes(case)
            views = [[flat[a:a + math.prod(t)].view(t) for a, t in zip(s["starts"], shapes)] for flat in (s["p"], s["g"])]
            s["opt"] = o = optim.AdamW(_context, *views, groups=[list(range(case["clients"]))] * len(shapes), lr=s["lr"], betas=(BETA1, BETA2),
                                       eps=ADAM_EPS, weight_decay=DECAY, max_norm=MAX_NORM if case["clip"] else None,
                                       state_bits=case["bits"], master=case["master"])
            o.steps.copy_(s["steps"])
            o.m.copy_(s["m"].view(-1))
            o.v.copy_(s["v"].view(-1))
            if case["bits"] == 8:
                o.m_scale.copy_(s["m_scale"].view(-1))
                o.v_scale.copy_(s["v_scale"].view(-1))
            if case["master"]:
                o.master.copy_(s["master"].view(-1))
            for k in ("m", "v", "m_scale", "v_scale", "master"):
                s.pop(k, None)
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
    if not s["case"]["p"]:
        return x.float()
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


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    v = _plain_dropout(s["x"], s)
    if c["residual"]:
        v = v + s["residual"].float()
    mean = v.mean(1, keepdim=True)
    d = v - mean
    rstd = (d.square().mean(1, keepdim=True) + EPS).rsqrt()
    out = [(d * rstd * s["weight"].float() + s["bias"].float()).to(dt)]
    if c["keep"] != "none":
        out.append(v.to(dt))
    return out + [mean[:, 0], rstd[:, 0]] if c["keep"] == "all" else out


def _plain_norm_backward(s):
    c, dt = s["case"], s["dy"].dtype
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["sum"].float() - s["mean"][:, None]) * rstd
    g = dy * s["weight"].float()
    ds = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if c["keep"] == "all":
        ds = ds + s["dsum"].float()
    grads = [(dy * xh).sum(0).to(dt), dy.sum(0).to(dt)]
    return [_plain_dropout(ds, s).to(dt)] + ([ds.to(dt)] if c["p"] else []) + grads


def _encode_m(m):
    a = m.abs().amax(1, keepdim=True)
    q = torch.sqrt((16129.0 * (m.abs() / a.clamp(min=1e-30)) - 0.25).clamp(min=0.0)).round()
    return (torch.sign(m) * q).to(torch.int8), a


def _encode_v(v):
    u = torch.sqrt(v)
    b = u.amax(1, keepdim=True)
    q = torch.sqrt((65025.0 * (u / b.clamp(min=1e-30)) - 0.25).clamp(min=0.0)).round()
    return torch.where(v > 0, q.clamp(min=1.0), 0.0).to(torch.uint8), b


def _decode_m(q, a):
    f = q.float()
    return f * f.abs() * (a / 16129.0)


def _decode_v(q, b):
    return (q.float().square() * (b / 65025.0)).square()


def _plain_adamw(s):
    c = s["case"]
    client, live = s["client"], s["active"]
    s["steps"] += live
    t = s["steps"].double()
    k1, k2 = (1 - BETA1 ** t).float(), (1 - BETA2 ** t).float()
    g = s["g"].view(-1, BLOCK).float() if s["aligned"] else torch.where(s["inside"], s["g"][s["at"]].float(), 0.0)
    out = {}
    if c["clip"]:
        square = g.square().sum(1, dtype=torch.float64)
        norm = torch.zeros(c["clients"], dtype=torch.float64, device="cuda").index_add_(0, client, square).sqrt()
        g = g * (MAX_NORM / norm).clamp(max=1.0).float()[client][:, None]
        out["norms"] = torch.where(live, norm, 0.0).float()
    if c["bits"] == 8:
        m0, v0 = _decode_m(s["m"], s["m_scale"]), _decode_v(s["v"], s["v_scale"])
    else:
        m0, v0 = s["m"], s["v"]
    m = BETA1 * m0 + (1 - BETA1) * g
    v = BETA2 * v0 + (1 - BETA2) * g.square()
    lr = s["rate"][client][:, None]
    w = s["master"] if c["master"] else s["p"].view(-1, BLOCK).float() if s["aligned"] else s["p"][s["at"]].float()
    new = w - lr * DECAY * w - lr * (m / k1[client][:, None]) / ((v / k2[client][:, None]).sqrt() + ADAM_EPS)
    step = live[client][:, None]
    if c["bits"] == 8:
        for name, (q, scale) in (("m", _encode_m(m)), ("v", _encode_v(v))):
            s[name] = torch.where(step, q, s[name])
            s[name + "_scale"] = torch.where(step, scale, s[name + "_scale"])
        s["m_out"].copy_(_decode_m(s["m"], s["m_scale"]))
        s["v_out"].copy_(_decode_v(s["v"], s["v_scale"]))
        out.update(m=s["m_out"].view(-1), v=s["v_out"].view(-1))
    else:
        s["m"], s["v"] = torch.where(step, m, m0), torch.where(step, v, v0)
        out.update(m=s["m"].view(-1), v=s["v"].view(-1))
    if c["master"]:
        s["master"] = torch.where(step, new, w)
        out["master"] = s["master"].view(-1)
    if s["aligned"]:
        p = s["p"].view(-1, BLOCK)
        p.copy_(torch.where(step, new.to(p.dtype), p))
    else:
        write = s["inside"] & step
        s["p"][s["at"][write]] = new[write].to(s["p"].dtype)
    return dict(out, p=s["p"], steps=s["steps"])


def run(s):
    c = s["case"]
    if own:
        from paper_2609_35352_gb300 import layernorm
        stream = torch.cuda.current_stream()
        if c["op"] == "norm":
            layernorm.layer_norm(s["ctx"], s["x"], s["out"], weight=s["weight"], bias=s["bias"], eps=EPS, residual=s.get("residual"),
                                 dropout=s["drop"], sum=s["sum"], mean=s["mean"], rstd=s["rstd"], stream=stream)
            return [s["out"]] + ([s["sum"]] if c["keep"] != "none" else []) + ([s["mean"], s["rstd"]] if c["keep"] == "all" else [])
        if c["op"] == "norm_backward":
            layernorm.layer_norm_backward(s["ctx"], s["dy"], s["sum"], s["mean"], s["rstd"], weight=s["weight"], dsum=s.get("dsum"),
                                          dropout=s["drop"], dx=s["dx"], dresidual=s["dresidual"], dweight=s["dweight"], dbias=s["dbias"],
                                          work=s["work"], stream=stream)
            return [s["dx"]] + ([s["dresidual"]] if c["p"] else []) + [s["dweight"], s["dbias"]]
        o = s["opt"]
        o.step(active=s["active"], stream=stream)
        out = {"p": s["p"], "steps": o.steps}
        if c["bits"] == 8:
            o.moments(s["m_out"], s["v_out"], stream=stream)
            out.update(m=s["m_out"].view(-1), v=s["v_out"].view(-1))
        else:
            out.update(m=o.m, v=o.v)
        if c["master"]:
            out["master"] = o.master
        if c["clip"]:
            out["norms"] = o.norms
        return out
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "adamw": _plain_adamw}[c["op"]](s)


# ----------------------------------------------------------------------------
# the definition in 64 bits
# ----------------------------------------------------------------------------
def _exact_dropout(x, c, s):
    """D(x) with the mask made on the host."""
    if not c["p"]:
        return x
    rows, cols = x.shape
    per_row = -(-cols // 4)
    with np.errstate(over="ignore"):
        n = np.arange(1, rows * per_row + 1, dtype=np.uint64) + np.uint64(s["rng_offset"])
        z = np.uint64(_key(s["rng_seed"])) + n * np.uint64(GOLDEN)
        z ^= z >> np.uint64(30)
        z *= np.uint64(MIX1)
        z ^= z >> np.uint64(27)
        z *= np.uint64(MIX2)
        z ^= z >> np.uint64(31)
    keep = z.astype("<u8").view("<u2").reshape(rows, 4 * per_row)[:, :cols] >= round(c["p"] * 65536)
    return torch.where(torch.from_numpy(keep).to(x.device), x * (65536 / (65536 - round(c["p"] * 65536))), 0.0)


def _exact_norm(c, s):
    v = _exact_dropout(s["x"].double(), c, s)
    if c["residual"]:
        v += s["residual"].double()
    mean = v.sum(1) / c["cols"]
    rstd = 1 / torch.sqrt(((v - mean[:, None]) ** 2).sum(1) / c["cols"] + EPS)
    y = (v - mean[:, None]) * rstd[:, None] * s["weight"].double() + s["bias"].double()
    return {"none": [y], "sum": [y, v], "all": [y, v, mean, rstd]}[c["keep"]]


def _exact_norm_backward(c, s):
    dy, n = s["dy"].double(), c["cols"]
    xh = (s["sum"].double() - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
    dweight, dbias = torch.einsum("tc,tc->c", dy, xh), dy.sum(0)
    g = dy * s["weight"].double()
    ds = g - g.sum(1, keepdim=True) / n - xh * (torch.einsum("tc,tc->t", g, xh) / n)[:, None]
    ds *= s["rstd"].double()[:, None]
    if c["keep"] == "all":
        ds += s["dsum"].double()
    dx = _exact_dropout(ds, c, s)
    return [dx, ds, dweight, dbias] if c["p"] else [dx, dweight, dbias]


def _exact_adamw(c, s):
    """Client by client and tensor by tensor."""
    shapes, clients = _shapes(c), c["clients"]
    p = s["p"].double()
    steps, active = s["steps"].tolist(), s["active"].tolist()
    m_all, v_all = torch.zeros(s["m"].numel(), dtype=torch.float64, device="cuda"), torch.zeros(s["m"].numel(), dtype=torch.float64, device="cuda")
    master = s["master"].double().view(-1) if c["master"] else None
    pieces, at = [[] for _ in range(clients)], 0
    for start, shape in zip(s["starts"].tolist(), shapes):
        n = math.prod(shape[1:])
        for i in range(clients):
            pieces[i].append((slice(start + i * n, start + (i + 1) * n), at, n))
            at += -(-n // BLOCK) * BLOCK
    norms = torch.zeros(clients, dtype=torch.float64, device="cuda")
    for i in range(clients):
        if c["clip"] and active[i]:
            norms[i] = math.sqrt(sum(float((s["g"][where].double() ** 2).sum()) for where, _, _ in pieces[i]))
        clip = MAX_NORM / max(MAX_NORM, float(norms[i]))
        t = steps[i] = steps[i] + active[i]
        for where, a, n in pieces[i]:
            nb = -(-n // BLOCK)
            inside = slice(a, a + n)
            if c["bits"] == 8:
                rows = slice(a // BLOCK, a // BLOCK + nb)
                q, r = s["m"][rows].double(), s["v"][rows].double()
                m = (q * q.abs() * s["m_scale"][rows].double() / 127 ** 2).view(-1)[:n]
                v = ((r * r * s["v_scale"][rows].double() / 255 ** 2) ** 2).view(-1)[:n]
            else:
                m, v = (s[k].view(-1)[inside].double() for k in ("m", "v"))
            if active[i]:
                g = s["g"][where].double() * clip
                m = m + (1 - BETA1) * (g - m)
                v = v + (1 - BETA2) * (g * g - v)
                w = master[inside] if c["master"] else p[where]
                w = (1 - s["lr"][i] * DECAY) * w - s["lr"][i] * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
                p[where] = w
                if c["master"]:
                    master[inside] = w
                if c["bits"] == 8:
                    m, v = _exact_packed(m, nb, 127), _exact_packed(v ** 0.5, nb, 255) ** 2
            m_all[inside], v_all[inside] = m, v
    out = {"p": p, "steps": torch.tensor(steps, device="cuda"), "m": m_all, "v": v_all}
    if c["master"]:
        out["master"] = master
    if c["clip"]:
        out["norms"] = norms
    return out


def _exact_packed(x, nb, top):
    """The nearest of the values q^2 / top^2 of the block's largest, by bisection among them."""
    full = torch.zeros(nb * BLOCK, dtype=torch.float64, device=x.device)
    full[:x.numel()] = x
    full = full.view(nb, BLOCK)
    most = full.abs().amax(1, keepdim=True)
    share = torch.where(most > 0, full.abs() / most, 0.0)
    values = (torch.arange(top + 1, dtype=torch.float64, device=x.device) / top) ** 2
    q = torch.bucketize(share, (values[1:] + values[:-1]) / 2)
    if top == 255:
        q = torch.where(share > 0, q.clamp(min=1), q)
    return (torch.sign(full) * values[q] * most).view(-1)[:x.numel()]


def exact(case, seed):
    return {"norm": _exact_norm, "norm_backward": _exact_norm_backward, "adamw": _exact_adamw}[case["op"]](case, _inputs(case, seed))
