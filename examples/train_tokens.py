"""Trains a next-token model whose token table is kept by the library: lookup, model, gradient by sorted tokens, global
norm over the model's gradients and the table's, clipping, update with difference propagation -- and a server lost half way.

    python examples/train_tokens.py [--steps 60]

The tokens follow a fixed rule with some noise (no data set is needed), so the loss falls quickly.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2104_01981_amd import Ecrm, Grads  # noqa: E402

VOCABULARY, DIM, K, SERVERS = 4096, 128, 4, 5
SEQUENCES, LENGTH = 64, 129
PAD = -1                                   # the tokens behind a sequence's end
MAX_NORM = 1.0


def batch(gen):
    """Sequences of different lengths: inputs and the tokens that follow them."""
    t = torch.empty(SEQUENCES, LENGTH, dtype=torch.int64, device="cuda")
    t[:, 0] = torch.randint(0, VOCABULARY, (SEQUENCES,), generator=gen, device="cuda")
    for i in range(1, LENGTH):
        noise = torch.rand(SEQUENCES, generator=gen, device="cuda") < 0.05
        other = torch.randint(0, VOCABULARY, (SEQUENCES,), generator=gen, device="cuda")
        t[:, i] = torch.where(noise, other, (5 * t[:, i - 1] + 7) % VOCABULARY)
    lengths = torch.randint(LENGTH // 2, LENGTH, (SEQUENCES, 1), generator=gen, device="cuda")
    inside = torch.arange(LENGTH - 1, device="cuda") < lengths
    tokens = torch.where(inside, t[:, :-1], PAD).flatten()
    follow = torch.where(inside, t[:, 1:], -100).flatten()
    return tokens, follow


def main(steps=60, verbose=True):
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = SEQUENCES * (LENGTH - 1)
    scale = DIM ** 0.5

    # the token table with its parities, and the context that keeps them
    E = torch.randn(VOCABULARY, DIM, generator=gen, device="cuda") * 0.02
    A = torch.zeros(VOCABULARY, DIM, device="cuda")
    PE, PA = torch.empty(VOCABULARY // K, DIM, device="cuda"), torch.empty(VOCABULARY // K, DIM, device="cuda")
    load = torch.zeros(2, SERVERS, dtype=torch.int64, device="cuda")
    ctx = Ecrm(VOCABULARY, DIM, K, SERVERS, lr=0.05, eps=1e-8, max_batch=n)
    scratch = torch.empty(ctx.scratch_bytes(), dtype=torch.uint8, device="cuda")
    ctx.bind(E, A, PE, PA, load[0], load[1], scratch)
    ctx.encode()

    # the model beside it, in 16 bits with 32-bit weights for its optimizer
    model = torch.nn.Linear(DIM, VOCABULARY, dtype=torch.bfloat16, device="cuda")
    with torch.no_grad():
        model.weight.copy_(torch.randn(VOCABULARY, DIM, generator=gen, device="cuda") * 0.02)
        model.bias.zero_()
    weights = [p.detach().float() for p in model.parameters()]
    squares = [torch.zeros_like(w) for w in weights]
    for p in model.parameters():
        p.grad = torch.zeros_like(p)

    # what a step leaves: one gradient row for each distinct token; the clipped gradients in 32 bits
    x = torch.zeros(n, DIM, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    rows, row_grads = torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(n, DIM, device="cuda")
    count, norm = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    clipped = [torch.empty_like(w) for w in weights]
    grads = Grads([p.grad for p in model.parameters()] + [(row_grads, count)])
    out = Grads(clipped + [row_grads])

    losses = []
    for step in range(steps):
        tokens, follow = batch(gen)
        lost = None
        if step == steps // 2:             # a server goes down; the lookup decodes its rows until it has been rebuilt
            lost = 2
            ctx.fail_server(lost)
        with torch.no_grad():
            ctx.embed(tokens, x, scale=scale, padding=PAD, lost_server=lost)
        if lost is not None:
            ctx.recover_server(lost)
        loss = torch.nn.functional.cross_entropy(model(x).float(), follow)
        x.grad = None
        for p in model.parameters():
            p.grad.zero_()
        loss.backward()

        ctx.embed_grad(tokens, x.grad, rows, row_grads, count, scale=scale, padding=PAD)
        grads.norm(norm)
        grads.clip(norm, MAX_NORM, out=out)
        ctx.update(rows, row_grads, n=int(count))
        with torch.no_grad():
            for p, w, s, g in zip(model.parameters(), weights, squares, clipped):
                s.addcmul_(g, g)
                w.addcdiv_(g, s.sqrt().add_(1e-8), value=-0.05)
                p.copy_(w)
        losses.append(float(loss.detach()))
        if verbose and (step % 10 == 0 or step == steps - 1 or lost is not None):
            print(f"step {step}: loss {losses[-1]:.3f}, norm {float(norm):.3f}, {int(count)} distinct tokens"
                  + (", one server down" if lost is not None else ""), flush=True)
    assert ctx.status() == 0
    drift = (PE.double() - E.double().view(-1, K, DIM).sum(1)).abs().max()
    if verbose:
        print(f"parities are off the sums of their entries by at most {float(drift):.1e}")
    return losses, float(drift)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    main(ap.parse_args().steps)
