"""A mask's state that nobody else holds stays its own until every stream has drawn from it: by itself, in the block and its gradients, in the
lookup and its gradients."""
import pytest
import torch

from paper_2104_01981_amd import Dropout, FeedForward
from test_gpu_dropout import PAD, Table, state, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls(kind, n=40, D=64, F=128):
    """A call of that kind with a mask and a stream, and what it writes."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, d = (torch.randn(n, D, generator=gen, device=DEV) for _ in range(2))
    out = torch.zeros(n, D, device=DEV)
    if kind == "apply":
        return (lambda drop, stream: drop.apply(x, out, stream=stream)), [out], ()
    if kind in ("forward", "backward"):
        weights = [torch.randn(*s, generator=gen, device=DEV) / 8 for s in ((F, D), (F, D), (D, F))]
        block = FeedForward(*weights, max_rows=n, training=True)
        if kind == "forward":
            return (lambda drop, stream: block.forward(x, out, dropout=drop, stream=stream)), [out], (block,)
        saved, grads = torch.randn(n, 2 * F, generator=gen, device=DEV), [torch.zeros_like(w) for w in weights]
        return (lambda drop, stream: block.backward(x, saved, d, out, *grads, dropout=drop, stream=stream)), [out] + grads, (block,)
    tab, keys = Table(1024, D, max_batch=n), tokens(1024, n, "text", 3)
    if kind == "embed":
        return (lambda drop, stream: tab.ctx.embed(keys, out, padding=PAD, dropout=drop, stream=stream)), [out], (tab,)
    if kind == "embed_grad_dense":
        dense = torch.zeros(1024, D, device=DEV)
        return (lambda drop, stream: tab.ctx.embed_grad_dense(keys, d, dense, padding=PAD, dropout=drop, stream=stream)), [dense], (tab,)
    names, count = torch.zeros(n, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    return (lambda drop, stream: tab.ctx.embed_grad(keys, d, names, out, count, padding=PAD, dropout=drop, stream=stream)), [out, names, count], (tab,)


@pytest.mark.parametrize("named", [True, False])
@pytest.mark.parametrize("kind", ["apply", "forward", "backward", "embed", "embed_grad", "embed_grad_dense"])
def test_a_state_that_is_dropped_before_a_stream_has_drawn_from_it(kind, named):
    call, outputs, _kept = calls(kind)
    call(Dropout(0.5, state(3, 4), 5), None)
    torch.cuda.synchronize()
    want = [o.clone() for o in outputs]
    for o in outputs:
        o.zero_()
    side, words = torch.cuda.Stream(), state(3, 4)
    drop, was = Dropout(0.5, words, 5), words.data_ptr()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        if not named:
            call(drop, None)                             # the current stream
    if named:
        call(drop, side)
    del drop, words
    again = [torch.full((2,), -1, dtype=torch.int64, device=DEV) for _ in range(64)]
    assert not side.query()                              # still held up
    assert was not in {t.data_ptr() for t in again}
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, want))
