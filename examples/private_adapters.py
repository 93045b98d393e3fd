"""Private adapters beside an encrypted, shared projection.

The server holds a frozen ternary projection that all clients share and evaluates
it under encryption (fiona_linear_eval): it sees neither activations nor results.
The side that holds the keys decrypts the projection's output and keeps what is a
client's own, the client's low-rank adapter and its training data:

    1. activations are packed by columns (ciphertext i: feature i of every token),
       encoded on the GPU and encrypted; the server evaluates y = W x;
    2. the adapters of all clients are trained at once on the decrypted
       activations: forward with dropout, the block's dropout, residual and layer
       norm in one call, a loss, backward through both, and an AdamW step in which
       each client is a model of its own (the norm's weights, shared, another); a
       client without data sits out;
    3. serving: one new token of each client, through projection, adapter and norm.

Run: python examples/private_adapters.py
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import oracle  # noqa: E402
from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import layernorm as LN  # noqa: E402
from paper_2609_35352_gb300 import optim as O  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

N, LIMBS, DELTA = 1024, 3, 2.0 ** 40
SLOTS = N // 2
WIDTH = 16
CLIENTS = 4


class KeyHolder:
    """Encrypts columns of activations and decrypts columns of results (secret
    key, evaluation form; encoding on the GPU, the rest in exact integers)."""

    def __init__(self, ctx, qs, rng):
        self.ctx, self.qs, self.rng = ctx, qs, rng
        self.s = self._ntt(rng.integers(-1, 2, (1, N)))[0]

    def _ntt(self, coeffs):
        out = torch.empty(coeffs.shape[0] * LIMBS * N, dtype=torch.int64, device="cuda")
        self.ctx.encode_coeffs(LIMBS, coeffs.shape[0],
                               torch.from_numpy(np.ascontiguousarray(coeffs, dtype=np.int64)).cuda(), out)
        return out.cpu().numpy().view(np.uint64).reshape(-1, LIMBS, N)

    def encode(self, columns):
        slots = torch.zeros(columns.shape[0], SLOTS, 2, dtype=torch.float64, device="cuda")
        slots[:, :, 0] = torch.from_numpy(columns).cuda()
        coeffs = torch.empty(columns.shape[0] * N, dtype=torch.int64, device="cuda")
        work = torch.empty(columns.shape[0] * N, dtype=torch.float64, device="cuda")
        out = torch.empty(columns.shape[0] * LIMBS * N, dtype=torch.int64, device="cuda")
        self.ctx.encode(LIMBS, columns.shape[0], slots, DELTA, coeffs, work, out)
        return out

    def encrypt(self, columns):
        n = columns.shape[0]
        m = self.encode(columns).cpu().numpy().view(np.uint64).reshape(n, LIMBS, N)
        e = self._ntt(np.rint(self.rng.normal(0.0, 3.2, (n, N))))
        ct = np.zeros((n, 2, LIMBS, N), np.uint64)
        for l, q in enumerate(self.qs):
            a = self.rng.integers(0, q, (n, N), dtype=np.uint64)
            ct[:, 1, l] = a
            ct[:, 0, l] = ((m[:, l].astype(object) + e[:, l] - a.astype(object) * self.s[l].astype(object)) % q).astype(np.uint64)
        return torch.from_numpy(ct.view(np.int64)).cuda()

    def decrypt(self, ct, scale):
        """[n][2][LIMBS][N] to columns [n][SLOTS]."""
        ct = ct.cpu().numpy().view(np.uint64).reshape(-1, 2, LIMBS, N)
        Q = 1
        for q in self.qs:
            Q *= q
        at = np.array([pow(5, j, 2 * N) for j in range(SLOTS)])
        columns = []
        for c in ct:
            total = np.zeros(N, dtype=object)
            for l, q in enumerate(self.qs):
                d = (c[0, l].astype(object) + c[1, l].astype(object) * self.s[l].astype(object)) % q
                v = np.array([int(x) for x in oracle.intt(np.array(d, dtype=np.uint64), q)], dtype=object)
                M = Q // q
                total = (total + v * (M * pow(M, -1, q))) % Q
            centred = np.array([float(x - Q if x > Q // 2 else x) for x in total])
            columns.append((np.fft.ifft(np.concatenate([centred, np.zeros(N)])) * (2 * N))[at].real / scale)
        return np.array(columns)


def shared_projection(ctx, rng):
    """A ternary layer W = gamma_j T_ji, compiled with shared signed sums."""
    signs = rng.integers(-1, 2, (WIDTH, WIDTH))
    gamma = rng.uniform(0.1, 0.3, WIDTH)
    routes = np.zeros((WIDTH, WIDTH), F.ROUTE_DTYPE)
    routes["kind"], routes["sign"] = W.TERM_TERNARY, signs
    routes["pt"] = np.arange(WIDTH)[:, None]  # gamma_j
    return F.Plan(ctx, F.compile_plan(WIDTH, WIDTH, WIDTH, routes)), signs * gamma[:, None], gamma


def normed(v):
    """What the clients want comes out of a norm too (weights one and zero)."""
    return torch.nn.functional.layer_norm(v, (WIDTH,))


def main(steps=300, verbose=True):
    say = print if verbose else (lambda *a: None)
    BUILD.build()
    oracle.build()
    rng = np.random.default_rng(2609)
    torch.manual_seed(2609)
    qs = W.ntt_primes(N, 40, LIMBS)
    ctx = F.Context(N, qs, device=0)
    keys = KeyHolder(ctx, qs, rng)
    plan, weights, gamma = shared_projection(ctx, rng)
    plaintexts = keys.encode(np.repeat(gamma[:, None], SLOTS, axis=1))

    def project(x):
        """y = x W^T [tokens][WIDTH], evaluated on ciphertexts."""
        columns = np.zeros((WIDTH, SLOTS))
        columns[:, :x.shape[0]] = x.double().cpu().numpy().T
        out = torch.empty(WIDTH * 2 * LIMBS * N, dtype=torch.int64, device="cuda")
        plan.eval(keys.encrypt(columns).reshape(-1), plaintexts, out, stream=torch.cuda.current_stream())
        y = keys.decrypt(out, DELTA ** 2)[:, :x.shape[0]].T
        return torch.from_numpy(np.ascontiguousarray(y)).float().cuda()

    # clients' tokens, one after another, and what each client wants on top of W
    counts = [200, 0, 180, 132]  # (the second has no data of its own)
    starts = [0] + [sum(counts[:i + 1]) for i in range(CLIENTS)]
    ranks, r_max = [4, 4, 8, 4], 8
    x = torch.randn(starts[-1], WIDTH, device="cuda")
    base = project(x)
    error = float((base.double() - x.double() @ torch.from_numpy(weights.T).cuda()).abs().max())
    say("encrypted projection: %d tokens, off by at most %.1e" % (starts[-1], error))
    shift = torch.randn(CLIENTS, WIDTH, 4, device="cuda") @ torch.randn(CLIENTS, 4, WIDTH, device="cuda") * 0.25
    target = x + base
    for c in range(CLIENTS):
        rows = slice(starts[c], starts[c + 1])
        target[rows] += x[rows] @ shift[c].T
    target = normed(target)

    # train all clients' adapters at once
    A = torch.randn(CLIENTS, r_max, WIDTH, device="cuda") * WIDTH ** -0.5
    B = torch.zeros(CLIENTS, WIDTH, r_max, device="cuda")
    batch = AD.Batch(ctx, starts, list(range(CLIENTS)), ranks, r_max, [2.0] * CLIENTS)
    work = batch.workspace(WIDTH, WIDTH, x.dtype)
    out, dx, h = torch.empty_like(base), torch.empty_like(x), torch.empty(starts[-1], r_max, device="cuda")
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    # the block's norm: residual + dropout(out), and what its gradient needs
    weight, bias = torch.ones(WIDTH, device="cuda"), torch.zeros(WIDTH, device="cuda")
    dweight, dbias = torch.empty_like(weight), torch.empty_like(bias)
    y, total, dy = torch.empty_like(base), torch.empty_like(base), torch.empty_like(base)
    mean, rstd = torch.empty(starts[-1], device="cuda"), torch.empty(starts[-1], device="cuda")
    norm_work = LN.workspace(ctx, *x.shape)
    # each client a group of its own, the norm's weights one more
    clients = list(range(CLIENTS))
    opt = O.AdamW(ctx, [A, B, weight, bias], [dA, dB, dweight, dbias], groups=[clients, clients, CLIENTS, CLIENTS],
                  lr=[2e-2] * CLIENTS + [2e-3], weight_decay=0.0, max_norm=1.0)
    active = torch.tensor([n > 0 for n in counts] + [True], device="cuda")
    idle = A[counts.index(0)].clone()
    drop, block_drop = AD.Dropout(0.02, seed=7), AD.Dropout(0.01, seed=8)
    stream, losses = torch.cuda.current_stream(), []
    for step in range(steps):
        batch.forward(x, A, B, out, base=base, h=h, dropout=drop, work=work, stream=stream)
        LN.layer_norm(ctx, out, y, weight=weight, bias=bias, residual=x, dropout=block_drop, sum=total, mean=mean, rstd=rstd, stream=stream)
        diff = y - target
        losses.append(float((diff * diff).mean()))
        LN.layer_norm_backward(ctx, diff * (2.0 / diff.numel()), total, mean, rstd, weight=weight, dropout=block_drop, dx=dy, dweight=dweight,
                               dbias=dbias, work=norm_work, stream=stream)
        batch.backward(x, h, dy, A, B, dx, dA, dB, dropout=drop, work=work, stream=stream)
        opt.lr.mul_(0.99)
        opt.step(active=active, stream=stream)
        drop, block_drop = drop.advance(*x.shape), block_drop.advance(*x.shape)
    if not torch.equal(A[counts.index(0)], idle):
        raise AssertionError("a client without data has another adapter than before")
    say("training: loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], steps))

    # serve one new token of each client
    token = torch.randn(CLIENTS, WIDTH, device="cuda")
    single = AD.Batch(ctx, list(range(CLIENTS + 1)), list(range(CLIENTS)), ranks, r_max, [2.0] * CLIENTS, gradients=False)
    served, stream_out = torch.empty(CLIENTS, WIDTH, device="cuda"), torch.empty(CLIENTS, WIDTH, device="cuda")
    token_base = project(token)
    single.forward(token, A, B, served, base=token_base, work=single.workspace(WIDTH, WIDTH, token.dtype), stream=stream)
    LN.layer_norm(ctx, served, stream_out, weight=weight, bias=bias, residual=token, stream=stream)
    trained = [c for c in range(CLIENTS) if counts[c]]
    wanted = normed(token + token_base + torch.stack([token[c] @ shift[c].T for c in range(CLIENTS)]))
    before = float((normed(token + token_base) - wanted)[trained].pow(2).mean())
    after = float((stream_out - wanted)[trained].pow(2).mean())
    say("serving: squared error on new tokens %.4f without adapters, %.4f with" % (before, after))
    return {"projection_error": error, "losses": losses, "before": before, "after": after}


if __name__ == "__main__":
    main()
