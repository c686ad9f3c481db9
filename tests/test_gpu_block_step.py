"""Lookup with dropout, the feed-forward block with dropout and a residual, their gradients down to the table's, as a training step runs
them, against the same step in 64 bits by automatic differentiation -- eagerly, and replayed from a graph.

In fp32 the kernels' errors are those of 32-bit sums: a gradient is off by at most a few hundred roundings (of 2^-24) of sums whose terms do
not cancel, 1e-4 of the gradient's own size (its Frobenius norm).  In 16 bits every value on the way is rounded once, half a step each, at
most eight of them one after the other (entries, h, y; b's terms, dg, du, d_x and the result): 8 half steps."""
import pytest
import torch

from paper_2104_01981_amd import Dropout, FeedForward
from test_gpu_dropout import PAD, Table, factors, half, state, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def close(got, want, share):
    off = float((got.double() - want).norm() / want.norm())
    assert off <= share, f"{off} of its size, {share} allowed"


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,D,F,kind", [(19, 128, 512, "silu"), (300, 64, 260, "gelu"), (1000, 132, 516, "silu")])
def test_step(n, D, F, kind, t):
    R, p, scale, seed = 4 * 256, 0.2, float(torch.tensor(D ** 0.5)), 31
    tab = Table(R, D, max_batch=n)
    tab.E.mul_(1.0 / float(tab.E.std()) / scale)
    g = torch.Generator(device=DEV).manual_seed(n)
    wg, wu, wd = (torch.randn(*s, generator=g, device=DEV).mul_(s[1] ** -0.5).to(t) for s in ((F, D), (F, D), (D, F)))
    target = torch.randn(n, D, generator=g, device=DEV)
    keys = tokens(R, n, "text", n)
    s = state(seed, 0)
    places = Dropout(p, s, 0), Dropout(p, s, 1)
    block = FeedForward(wg, wu, wd, max_rows=n, activation=kind, training=True)
    x, y, d_y, d_x = (torch.zeros(n, D, dtype=t, device=DEV) for _ in range(4))
    saved, grads = torch.zeros(n, 2 * F, dtype=t, device=DEV), [torch.zeros_like(w) for w in (wg, wu, wd)]
    dense = torch.zeros(R, D, device=DEV)

    def step():
        tab.ctx.embed(keys, x, scale=scale, padding=PAD, dropout=places[0])
        block.forward(x, y, residual=x, dropout=places[1], saved=saved)
        torch.sub(y, target.to(t), out=d_y)              # the gradient of half the squared distance
        block.backward(x, saved, d_y, d_x, *grads, add=d_y, dropout=places[1])
        tab.ctx.embed_grad_dense(keys, d_x, dense, scale=scale, padding=PAD, dropout=places[0])
        s[1] += 2

    def check(number):
        E, *w = (v.double().requires_grad_() for v in (tab.E, wg, wu, wd))
        found = (keys != PAD)[:, None].double()
        a = E[keys.clamp(min=0)] * scale * found * factors(p, seed, number, n, D)
        gate, up = a @ w[0].t(), a @ w[1].t()
        act = torch.nn.functional.silu(gate) if kind == "silu" else torch.nn.functional.gelu(gate)
        z = a + (act * up) @ w[2].t() * factors(p, seed, number + 1, n, D)
        (0.5 * (z - target.double()) ** 2).sum().backward()
        share = 1e-4 if t == torch.float32 else 8 * half(t)
        for got, want in zip([y, dense] + grads, [z, E.grad] + [v.grad for v in w]):
            close(got, want.detach(), share)

    step()
    check(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        check(4 + 2 * i)
    assert tab.ctx.status() == 0
