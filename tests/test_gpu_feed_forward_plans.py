"""The gated feed-forward block, exactly, at sizes that take the plans which those of test_gpu_feed_forward.py do not take; and gradients in the
place of the output's gradient, where the order of the launches matters, at the sizes of both.  Small whole numbers: results are the reference's bits.

Together the sizes take every kind of launch that a block on 256 CUs may have (tests/test_ffn_plan.py asks the planner)."""
import pytest
import torch

import test_gpu_feed_forward as ff
from paper_2104_01981_amd import Dropout, FeedForward
from test_gpu_dropout import factors, state

pytestmark = pytest.mark.gpu
# parts of K joined by several workgroups of few rows; last rows of every product in every tile and, of 16 bits, by the few rows' kernel, with and
# without parts; gradients side by side in every tile, with either, both or none of the two cut along K
PLANNED = [(1, 4, 1956), (18, 4, 1924), (1379, 7412, 4), (1729, 624, 620), (17566, 2760, 12), (53645, 332, 132), (53788, 120, 296),
           (8324, 120, 2620), (32796, 1748, 84), (8217, 68, 4608), (7048, 492, 1700), (10753, 2168, 700), (98217, 352, 484), (3109, 6720, 1176),
           (54334, 116, 2392), (1494, 3564, 7040), (97882, 1148, 340), (1424, 3876, 9668), (81828, 1472, 424), (81244, 880, 1280)]

# the largest and smallest widths beside each other, in the few rows' kernel and in tiles
WIDEST = [(1, 65536, 4), (40, 65536, 8), (300, 65536, 12), (1, 4, 65536), (40, 4, 65536), (300, 12, 65536), (17, 32768, 64)]


@pytest.mark.parametrize("t", ff.TYPES)
@pytest.mark.parametrize("n,D,F", PLANNED + WIDEST)
def test_forward_exactly(n, D, F, t):
    ff.test_forward_exactly(n, D, F, t)


@pytest.mark.parametrize("t", ff.TYPES)
@pytest.mark.parametrize("n,D,F", PLANNED + WIDEST)
def test_backward_exactly(n, D, F, t):
    ff.test_backward_exactly(n, D, F, t)


@pytest.mark.parametrize("t", ff.TYPES)
@pytest.mark.parametrize("n,D,F", ff.SIZES + ff.LARGE + PLANNED + WIDEST)
def test_gradients_in_the_place_of_the_outputs(n, D, F, t):
    """d_x takes the place of what the weights' gradients read: d_x behind them without a mask, in two launches that share parts and
    counters; beside them with one, which leaves them a copy.  It may also be what d_x is added to, alone."""
    extra = 4
    gen, x, wg, wu, wd = ff.exact_case(n, D, F, t, extra, 5 * n + D + F)
    g, u, h, _ = ff.relu_reference(x, wg, wu, wd)
    saved = torch.cat([g, u], 1).to(t)
    d = ff.whole(n, D, t, gen, min(1.0, 6.0 / D), extra)
    block = FeedForward(wg, wu, wd, max_rows=n, activation="relu", training=True)
    for p in (None, 0.5):
        drop = Dropout(p, state(80, 9), n) if p is not None else None
        e = d.double() * factors(p, 80, 9 + n, n, D) if p is not None else d.double()
        b = e @ wd.double()
        dg, du = b * u * (g > 0), b * g.clamp(min=0)
        assert float(torch.stack([dg.abs().max(), du.abs().max(), h.abs().max()]).max()) <= 256     # exact in every type
        want_x = dg @ wg.double() + du @ wu.double()
        want = [w.to(t) for w in (dg.t() @ x.double(), du.t() @ x.double(), e.t() @ h)]

        def run(d_out, d_x, add):
            grads = [torch.full(s, -7.0, dtype=t, device=ff.DEV) for s in ((F, D), (F, D), (D, F))]
            ff.poisoned(block).backward(x, saved, d_out, d_x, *grads, add=add, dropout=drop)
            assert torch.equal(d_x, (want_x + add_was if add is not None else want_x).to(t)), (p, int((d_x != want_x.to(t)).sum()))
            for got, w in zip(grads, want):
                assert torch.equal(got, w), (p, int((got != w).sum()))

        add_was = d.double()
        for added in (False, True):                      # the output's gradient's place, as such and with that added
            c, around = ff.inside(n, D, t, extra)
            c.copy_(d)
            run(c, c, c if added else None)
            assert ff.untouched(around, n, D)
        c, around = ff.inside(n, D, t, extra)            # the place of what is added alone
        add_was = ff.whole(n, D, t, gen, 0.5, extra).double()
        c.copy_(add_was)
        run(d, c, c)
        assert ff.untouched(around, n, D)


def test_the_most_rows():
    """2^26 rows, of the smallest width: a million tiles, sums over a million tiles of K, rows of the workspace up to 24 GiB from the first."""
    n, D, F, t, p = 1 << 26, 4, 4, torch.bfloat16, 0.5
    free, _ = torch.cuda.mem_get_info()
    if free < 200 << 30:
        pytest.skip("not enough device memory")
    gen = torch.Generator(device=ff.DEV).manual_seed(1)

    def some(*shape):
        return torch.randint(-1, 2, shape, generator=gen, device=ff.DEV, dtype=torch.int8).to(t)

    x, d, wg, wu, wd = some(n, D), some(n, D), some(F, D), some(F, D), some(D, F)
    block = FeedForward(wg, wu, wd, max_rows=n, activation="relu", training=True)
    out, saved, d_x = torch.full_like(x, -7.0), torch.full((n, 2 * F), -7.0, dtype=t, device=ff.DEV), torch.full_like(x, -7.0)
    drop = Dropout(p, state(81, 10), 1)
    block.forward(x, out, residual=x, dropout=drop, saved=saved)
    for accumulate in (False, True):
        wide = [torch.full(s, 3.0, device=ff.DEV) for s in ((F, D), (F, D), (D, F))]
        block.backward(x, saved, d, d_x, *wide, add=d, dropout=drop, accumulate=accumulate)
        if not accumulate:
            first = wide
    kept = torch.ones_like(x)                            # its masks are held to their definition by test_gpu_dropout.py
    drop.apply(kept, kept)
    want = [torch.zeros(s, dtype=torch.float64, device=ff.DEV) for s in ((F, D), (F, D), (D, F))]
    for i in range(0, n, 1 << 22):
        at = slice(i, i + (1 << 22))
        g, u, h, y = ff.relu_reference(x[at], wg, wu, wd)
        m, e = kept[at].double(), kept[at].double() * d[at].double()
        assert torch.equal(saved[at], torch.cat([g, u], 1).to(t)) and torch.equal(out[at], (y * m + x[at].double()).to(t)), i
        b = e @ wd.double()
        dg, du = b * u * (g > 0), b * g.clamp(min=0)
        assert float(torch.stack([dg.abs().max(), du.abs().max(), h.abs().max()]).max()) <= 256
        assert torch.equal(d_x[at], (dg @ wg.double() + du @ wu.double() + d[at].double()).to(t)), i
        for w, left, right in zip(want, (dg, du, e), (x[at].double(), x[at].double(), h)):
            w += (left[:, :, None] * right[:, None, :]).sum(0)
    assert max(float(w.abs().max()) for w in want) < 1 << 24                       # exact in sums of 32 bits
    assert all(torch.equal(a.double(), w) and torch.equal(b.double(), w + 3) for a, b, w in zip(first, wide, want))
