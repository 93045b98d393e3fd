"""A training step as it is used: adapters beside a projection, the block's dropout,
residual and layer norm, the gradient back through both, and an AdamW step in which every
client is a model of its own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2609_35352_gb300 import adapters as AD  # noqa: E402
from paper_2609_35352_gb300 import build as BUILD  # noqa: E402
from paper_2609_35352_gb300 import fiona as F  # noqa: E402
from paper_2609_35352_gb300 import layernorm as LN  # noqa: E402
from paper_2609_35352_gb300 import optim as O  # noqa: E402
from paper_2609_35352_gb300 import workloads as W  # noqa: E402

import optim_util as OU  # noqa: E402
from adapter_util import factor_of, keep_mask  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    BUILD.build()
    return F.Context(1024, W.ntt_primes(1024, 50, 1), device=0)


CLIENTS, COUNTS, RANKS, R, WIDTH = 4, [50, 0, 70, 41], [8, 4, 8, 5], 8, 96


class Block:
    def __init__(self, ctx, dtype, state_bits, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

        self.ctx, T = ctx, sum(COUNTS)
        self.starts = [0] + [sum(COUNTS[:i + 1]) for i in range(CLIENTS)]
        self.x, self.base, self.residual, self.target = (normal(T, WIDTH) for _ in range(4))
        self.A, self.B = normal(CLIENTS, R, WIDTH, scale=WIDTH ** -0.5), normal(CLIENTS, WIDTH, R, scale=0.3)
        self.weight, self.bias = torch.ones(WIDTH, device="cuda") * 1.1, torch.zeros(WIDTH, device="cuda") + 0.1
        self.batch = AD.Batch(ctx, self.starts, list(range(CLIENTS)), RANKS, R, [2.0, 1.0, 0.5, 1.0])
        self.work, self.norm_work = self.batch.workspace(WIDTH, WIDTH, dtype), LN.workspace(ctx, T, WIDTH)
        self.out, self.y, self.total, self.dout, self.dx, self.dresidual = (torch.empty_like(self.x) for _ in range(6))
        self.h = torch.empty(T, R, device="cuda")
        self.mean, self.rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        self.grads = [torch.empty_like(t) for t in (self.A, self.B, self.weight, self.bias)]
        self.drop, self.block_drop = AD.Dropout(0.1, 3, 1 << 35), AD.Dropout(0.2, 4)
        clients = list(range(CLIENTS))
        self.opt = O.AdamW(ctx, [self.A, self.B, self.weight, self.bias], self.grads, groups=[clients, clients, CLIENTS, CLIENTS],
                           lr=1e-2, max_norm=0.05, state_bits=state_bits, master=dtype != torch.float32)
        self.active = torch.tensor([n > 0 for n in COUNTS] + [True], device="cuda")
        self.dy = torch.empty_like(self.x)

    def step(self):
        s = torch.cuda.current_stream()
        self.batch.forward(self.x, self.A, self.B, self.out, base=self.base, h=self.h, dropout=self.drop, work=self.work, stream=s)
        LN.layer_norm(self.ctx, self.out, self.y, weight=self.weight, bias=self.bias, residual=self.residual, dropout=self.block_drop,
                      sum=self.total, mean=self.mean, rstd=self.rstd, stream=s)
        torch.sub(self.y, self.target, out=self.dy)
        LN.layer_norm_backward(self.ctx, self.dy, self.total, self.mean, self.rstd, weight=self.weight, dropout=self.block_drop, dx=self.dout,
                               dresidual=self.dresidual, dweight=self.grads[2], dbias=self.grads[3], work=self.norm_work, stream=s)
        self.batch.backward(self.x, self.h, self.dout, self.A, self.B, self.dx, self.grads[0], self.grads[1], dropout=self.drop,
                            work=self.work, stream=s)
        self.opt.step(active=self.active, stream=s)

    def state(self):
        o = self.opt
        return [t.clone() for t in (self.A, self.B, self.weight, self.bias, self.dx, self.dresidual, o.m, o.v, o.steps, o.norms)]


def test_gradients_against_autograd_in_64_bits(ctx):
    """fp32: every gradient of the block within 1000 roundings (the sums forward and back have
    some 500 terms one after another, each rounded in a product and an addition)."""
    b = Block(ctx, torch.float32, 32)
    before = [t.double().cpu() for t in (b.A, b.B, b.weight, b.bias)]
    b.step()
    torch.cuda.synchronize()
    leaves = [t.double().cpu().requires_grad_() for t in (b.x, b.residual)] + [t.clone().requires_grad_() for t in before]
    x, residual, A, B, weight, bias = leaves
    keep = [torch.from_numpy(keep_mask(x.shape[0], WIDTH, d.p, d.seed, d.offset)) * factor_of(d.p) for d in (b.drop, b.block_drop)]
    out = []
    for c in range(CLIENTS):
        rows = slice(b.starts[c], b.starts[c + 1])
        k = RANKS[c]
        out.append(b.base.double().cpu()[rows] + [2.0, 1.0, 0.5, 1.0][c] * ((x * keep[0])[rows] @ A[c, :k].T) @ B[c, :, :k].T)
    y = torch.nn.functional.layer_norm(residual + torch.cat(out) * keep[1], (WIDTH,), weight, bias, 1e-5)
    (0.5 * (y - b.target.double().cpu()).square()).sum().backward()
    for name, leaf, got in zip(("dx", "dresidual", "dA", "dB", "dweight", "dbias"), leaves, [b.dx, b.dresidual] + b.grads):
        off = (got.double().cpu() - leaf.grad).norm() / leaf.grad.norm()
        assert off <= 1000 * 2.0 ** -24, (name, float(off))
    # and the step that they make
    g = [t.grad.numpy() for t in leaves[2:]]
    settings = OU.Group(1e-2, max_norm=0.05)
    for c in (0, 2, 3):
        norm = OU.norm_of([g[0][c], g[1][c]])
        assert norm > 0.05 and abs(float(b.opt.norms[c]) / norm - 1) < 1000 * 2.0 ** -24
        for i, new in ((0, b.A), (1, b.B)):
            kernel = b.grads[i][c].double().cpu().numpy()
            (w, dw), _, _ = OU.step(settings, 1, before[i][c].numpy(), np.zeros_like(kernel), np.zeros_like(kernel), kernel,
                                    OU.norm_of([b.grads[j][c].double().cpu().numpy() for j in (0, 1)]))
            OU.check("weights", "f32", new[c].double().cpu().numpy(), w, dw)
    assert torch.equal(b.A[1].double().cpu(), before[0][1]) and torch.equal(b.B[1].double().cpu(), before[1][1])
    assert b.opt.steps.tolist() == [1, 0, 1, 1, 1]


@pytest.mark.parametrize("state_bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_captured_steps_are_the_eager_ones(ctx, dtype, state_bits):
    eager, captured = Block(ctx, dtype, state_bits), Block(ctx, dtype, state_bits)
    for _ in range(5):
        eager.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager.state(), captured.state()))
    assert all(torch.isfinite(t.float()).all() for t in eager.state())
    # two blocks' steps on two streams at once, each with workspaces of its own
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        for s, b in ((one, eager), (two, captured)):
            with torch.cuda.stream(s):
                b.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager.state(), captured.state()))
