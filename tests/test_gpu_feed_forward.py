"""The gated feed-forward block and its gradients (ecrm_ffn_forward, ecrm_ffn_backward) against plain 64-bit forms.

First with small whole numbers and the activation max(g, 0), where every sum, product and rounding between the products is exact, so
that the results are the reference's bits: sizes around what a chunk, a block, a tile and a part of K take, strides, and values that
are not finite everywhere around the operands and in the workspace.  Then with values as a model has them and a bound for each error:

    h = act(g) u rounded to the type: half a step of h, and what g and u are off by, times the activation's and its derivative's
    bounds (|act(g)| <= |g|, |act'| <= 1.13, |act''| <= 1);  a sum of K terms in 32 bits, each addition off by at most a
    step (2^-23): K 2^-23 times the sum of the absolute terms;  activations 2^-19 max(1, |g|)."""
import pytest
import torch

import philox
from paper_2104_01981_amd import ECRM_EBATCH, ECRM_EINVAL, ECRM_ESCRATCH, Dropout, EcrmError, FeedForward
from test_gpu_dropout import factors, half, state

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 4, 4), (1, 128, 512), (2, 12, 20), (3, 8, 132), (5, 60, 64), (15, 64, 68), (16, 68, 60), (17, 132, 36), (31, 36, 260), (33, 256, 100),
         (63, 100, 256), (65, 128, 128), (128, 124, 516), (129, 260, 124), (257, 64, 1028), (300, 516, 268), (1000, 4, 512), (1025, 128, 4)]
# every tiling of every product, of 16 and of 32 bits; of their kinds of launches -- cut along K or not, rows behind the last whole tiles -- 91 of
# 131, the others at the sizes of test_gpu_feed_forward_plans.py
LARGE = [(2100, 512, 1028), (4099, 260, 2052), (300, 1024, 4096), (3000, 1024, 1028), (5000, 512, 2052), (8300, 132, 1028), (16400, 1024, 260),
         (4100, 1024, 4100), (95597, 84, 92), (685, 1900, 860), (652, 6152, 364), (58412, 1152, 4), (370, 7080, 108), (26758, 36, 1272),
         (163, 7060, 1756), (5180, 1268, 956), (2932, 1208, 1664)]


def whole(n, m, t, gen, share, extra=0):
    """Numbers -1, 0, 1 inside wider rows of NaN, a row of it behind; from a multiple of four elements on, not always of 16 bytes."""
    wide = torch.full((n + 1, m + extra), float("nan"), dtype=t, device=DEV)
    x = torch.randint(-1, 2, (n, m), generator=gen, device=DEV) * (torch.rand(n, m, generator=gen, device=DEV) < share)
    wide[:n, extra:] = x.to(t)
    return wide[:n, extra:]


def inside(n, m, t, extra):
    wide = torch.full((n + 1, m + extra), -7.0, dtype=t, device=DEV)
    return wide[:n, extra:], wide


def untouched(wide, n, m):
    return bool((wide[n] == -7.0).all()) and bool((wide[:, :wide.shape[1] - m] == -7.0).all())


def behind(n, m, t, extra, fill):
    """Contiguous, `extra` elements from the begin of its memory."""
    flat = torch.full((n * m + extra + 8,), fill, dtype=t, device=DEV)
    return flat[extra:extra + n * m].view(n, m), flat


def relu_reference(x, wg, wu, wd):
    x, wg, wu, wd = x.double(), wg.double(), wu.double(), wd.double()
    g, u = x @ wg.t(), x @ wu.t()
    h = g.clamp(min=0) * u
    return g, u, h, h @ wd.t()


def poisoned(block):
    block.workspace.fill_(255)                           # not a number, in every type
    return block


def exact_case(n, D, F, t, extra, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    share = min(1.0, 6.0 / D)                            # about four terms to a sum
    x = whole(n, D, t, gen, 1.0, extra)
    wg, wu = whole(F, D, t, gen, share, extra), whole(F, D, t, gen, share, 2 * extra)
    wd = whole(D, F, t, gen, min(1.0, 6.0 / F), extra)
    return gen, x, wg, wu, wd


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,D,F", SIZES + LARGE)
def test_forward_exactly(n, D, F, t):
    for extra in (0, 4, 8):
        gen, x, wg, wu, wd = exact_case(n, D, F, t, extra, n + D + F)
        g, u, h, y = relu_reference(x, wg, wu, wd)
        assert float(h.abs().max()) <= 256                # exact in every type
        block = poisoned(FeedForward(wg, wu, wd, max_rows=n + 3, activation="relu"))
        r = whole(n, D, t, gen, 0.5, extra)
        for residual, p in ((None, None), (r, None), (r, 0.5)):
            out, around = inside(n, D, t, extra)
            saved, saved_around = behind(n, 2 * F, t, extra, -7.0)
            want = y
            if p is not None:                             # the factor is 2
                want = want * factors(p, 77, 5 + n, n, D)
            if residual is not None:
                want = want + residual.double()
            drop = Dropout(p, state(77, 5), n) if p is not None else None
            block.forward(x, out, residual=residual, dropout=drop, saved=saved)
            assert torch.equal(out, want.to(t)), (extra, p, int((out != want.to(t)).sum()))
            assert torch.equal(saved, torch.cat([g, u], 1).to(t))
            assert untouched(around, n, D)
            assert bool((saved_around[:extra] == -7.0).all()) and bool((saved_around[extra + n * 2 * F:] == -7.0).all())
            again, _ = inside(n, D, t, 0)
            poisoned(block).forward(x, again, residual=residual, dropout=drop)
            assert torch.equal(again, out)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,D,F", SIZES + LARGE)
def test_backward_exactly(n, D, F, t):
    for extra, p in ((0, None), (4, 0.5), (8, None)):
        gen, x, wg, wu, wd = exact_case(n, D, F, t, extra, 3 * n + D + F)
        g, u, h, _ = relu_reference(x, wg, wu, wd)
        saved, _ = behind(n, 2 * F, t, extra, float("nan"))
        saved.copy_(torch.cat([g, u], 1))
        d = whole(n, D, t, gen, min(1.0, 6.0 / D), extra)
        drop = Dropout(p, state(78, 6), n) if p is not None else None
        e = d.double() * factors(p, 78, 6 + n, n, D) if p is not None else d.double()
        b = e @ wd.double()
        dg, du = b * u * (g > 0), b * g.clamp(min=0)
        assert float(torch.stack([dg.abs().max(), du.abs().max(), h.abs().max()]).max()) <= 256
        want_x = dg @ wg.double() + du @ wu.double()
        want = [dg.t() @ x.double(), du.t() @ x.double(), e.t() @ h]
        block = poisoned(FeedForward(wg, wu, wd, max_rows=n, activation="relu", training=True))
        for add in (None, d):
            d_x, around = inside(n, D, t, extra)
            grads, grads_around = zip(*[behind(*s, t, extra, -7.0) for s in ((F, D), (F, D), (D, F))])
            block.backward(x, saved, d, d_x, *grads, add=add, dropout=drop)
            assert torch.equal(d_x, (want_x + add.double() if add is not None else want_x).to(t)) and untouched(around, n, D)
            for got, w, flat in zip(grads, want, grads_around):
                assert torch.equal(got, w.to(t))
                assert bool((flat[:extra] == -7.0).all()) and bool((flat[extra + D * F:] == -7.0).all())
        # in the type, added to what is there
        poisoned(block).backward(x, saved, d, None, *grads, dropout=drop, accumulate=True)
        for got, w in zip(grads, want):
            assert torch.equal(got, (w.to(t).double() + w).to(t))
        # in 32 bits, added to what is there; the input's gradient alone; the weights' alone; in the place of the output's gradient
        wide = [torch.full(s, 3.0, device=DEV) for s in ((F, D), (F, D), (D, F))]
        poisoned(block).backward(x, saved, d, None, *wide, dropout=drop, accumulate=True)
        for got, w in zip(wide, want):
            assert torch.equal(got, (w + 3).float())
        alone, _ = inside(n, D, t, 0)
        poisoned(block).backward(x, saved, d, alone, dropout=drop)
        assert torch.equal(alone, want_x.to(t))
        poisoned(block).backward(x, saved, d, d, add=d, dropout=drop)
        assert torch.equal(d, d_x)


# ---- values as a model has them --------------------------------------------------------------------------------------------
def value(kind, g):
    if kind == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * torch.special.erfc(-g * 0.5 ** 0.5) if kind == "gelu" else g.clamp(min=0)


def slope(kind, g):
    if kind == "silu":
        q = torch.sigmoid(g)
        return q + g * q * torch.sigmoid(-g)
    if kind == "gelu":
        return 0.5 * torch.special.erfc(-g * 0.5 ** 0.5) + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    return (g > 0).double()


STEP, FUNCTION = 2.0 ** -23, 2.0 ** -19


def model(n, D, F, t, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, D, generator=gen, device=DEV).to(t)
    wg = (2 * torch.randn(F, D, generator=gen, device=DEV) * D ** -0.5).to(t)
    wu = (torch.randn(F, D, generator=gen, device=DEV) * D ** -0.5).to(t)
    wd = (torch.randn(D, F, generator=gen, device=DEV) * F ** -0.5).to(t)
    return gen, x, wg, wu, wd


def off(got, want, tol):
    bad = (got.double() - want).abs() > tol
    return f"{int(bad.sum())} of {bad.numel()}, {float(((got.double() - want).abs() / tol).max())} times the bound" if bool(bad.any()) else ""


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("n,D,F,p", [(1, 128, 512, None), (7, 256, 1024, None), (19, 1024, 260, 0.1), (600, 128, 512, 0.1), (777, 260, 684, 0.3)])
def test_forward(n, D, F, p, kind, t):
    gen, x, wg, wu, wd = model(n, D, F, t, n + F)
    r = torch.randn(n, D, generator=gen, device=DEV).to(t)
    out, saved = torch.empty_like(x), torch.empty(n, 2 * F, dtype=t, device=DEV)
    drop = Dropout(p, state(1, 2), 3) if p else None
    FeedForward(wg, wu, wd, max_rows=n, activation=kind).forward(x, out, residual=r, dropout=drop, saved=saved)
    X, G, U, W = (v.double() for v in (x, wg, wu, wd))
    g, u = X @ G.t(), X @ U.t()
    eg, eu = D * STEP * (X.abs() @ G.abs().t()), D * STEP * (X.abs() @ U.abs().t())
    assert not off(saved[:, :F], g, half(t) * (g.abs() + eg) + eg + 1e-7)
    assert not off(saved[:, F:], u, half(t) * (u.abs() + eu) + eu + 1e-7)
    h = value(kind, g) * u
    eh = 1.13 * eg * u.abs() + (value(kind, g).abs() + eg * 1.13) * eu + FUNCTION * g.abs().clamp(min=1) * u.abs()
    eh = eh + half(t) * (h.abs() + eh) + 1e-7             # and what is below fp16's normal values: at most 2^-25
    m = factors(p, 1, 5, n, D) if p else torch.ones((), dtype=torch.float64, device=DEV)
    y = (h @ W.t()) * m
    ey = (eh @ W.abs().t() + F * STEP * (h.abs() + eh) @ W.abs().t()) * m + 2 * STEP * y.abs()
    want = y + r.double()
    assert not off(out, want, ey + (half(t) + STEP) * (want.abs() + ey) + 1e-7)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("n,D,F,p", [(1, 128, 512, None), (600, 128, 512, 0.1), (777, 260, 684, 0.3), (2500, 64, 256, 0.1)])
def test_backward(n, D, F, p, kind, t):
    gen, x, wg, wu, wd = model(n, D, F, t, n + F)
    X, G, U, W = (v.double() for v in (x, wg, wu, wd))
    saved = torch.cat([X @ G.t(), X @ U.t()], 1).to(t)
    g, u = saved.double().split(F, 1)
    d = torch.randn(n, D, generator=gen, device=DEV).to(t)
    m = factors(p, 1, 5, n, D) if p else torch.ones((), dtype=torch.float64, device=DEV)
    d_x = torch.empty_like(x)
    grads = [torch.empty_like(w) for w in (wg, wu, wd)]
    wide = [torch.empty(w.shape, device=DEV) for w in (wg, wu, wd)]
    block = FeedForward(wg, wu, wd, max_rows=n, activation=kind, training=True)
    drop = Dropout(p, state(1, 2), 3) if p else None
    block.backward(x, saved, d, d_x, *grads, add=d, dropout=drop)
    block.backward(x, saved, d, None, *wide, dropout=drop)
    e = d.double() * m
    ee = (half(t) + 2 * STEP) * e.abs() if p else 0 * e.abs()
    b = e @ W
    eb = ee @ W.abs() + D * STEP * ((e.abs() + ee) @ W.abs())
    a, s = value(kind, g), slope(kind, g)
    fn = FUNCTION * g.abs().clamp(min=1)
    dg, du, h = b * u * s, b * a, a * u
    edg = eb * (u * s).abs() + (b.abs() + eb) * u.abs() * fn
    edu = eb * a.abs() + (b.abs() + eb) * fn
    eh = fn * u.abs()
    edg, edu, eh = (v + (half(t) + 2 * STEP) * (w.abs() + v) + 1e-7 for v, w in ((edg, dg), (edu, du), (eh, h)))
    want = dg @ G + du @ U + d.double()
    tol = edg @ G.abs() + edu @ U.abs() + 2 * F * STEP * ((dg.abs() + edg) @ G.abs() + (du.abs() + edu) @ U.abs())
    assert not off(d_x, want, tol + (half(t) + STEP) * (want.abs() + tol) + 1e-7)
    for got, in32, left, e_left, right, e_right in ((grads[0], wide[0], dg, edg, X, 0 * X), (grads[1], wide[1], du, edu, X, 0 * X),
                                                    (grads[2], wide[2], e, ee, h, eh)):
        want = left.t() @ right
        tol = e_left.t() @ right.abs() + (left.abs() + e_left).t() @ e_right
        tol = tol + n * STEP * ((left.abs() + e_left).t() @ (right.abs() + e_right))
        assert not off(in32, want, tol + STEP * want.abs() + 1e-30)
        assert not off(got, want, tol + half(t) * (want.abs() + tol) + 1e-7)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gradients_against_differences(kind):
    """Central differences of a 64-bit forward pass along random directions: their own error is about step^2 and 2^-53 / step relative
    to sums of this size, below 1e-7 of the sum of the absolute terms; the gradients' is that of 32-bit sums, (n + D + F) 2^-23."""
    n, D, F, p = 37, 60, 100, 0.25
    gen, x, wg, wu, wd = model(n, D, F, torch.float32, 9)
    d = torch.randn(n, D, generator=gen, device=DEV)
    m = factors(p, 1, 5, n, D)
    drop, saved, out = Dropout(p, state(1, 2), 3), torch.empty(n, 2 * F, device=DEV), torch.empty_like(x)
    block = FeedForward(wg, wu, wd, max_rows=n, activation=kind, training=True)
    block.forward(x, out, residual=x, dropout=drop, saved=saved)
    got = [torch.empty_like(v) for v in (x, wg, wu, wd)]
    block.backward(x, saved, d, *got, add=d, dropout=drop)

    def loss(x, wg, wu, wd):
        return (d.double() * (x + (value(kind, x @ wg.t()) * (x @ wu.t())) @ wd.t() * m)).sum()

    at = [v.double() for v in (x, wg, wu, wd)]
    for i in range(4):
        along = torch.randn(at[i].shape, generator=gen, device=DEV, dtype=torch.float64)
        step = 1e-5
        ends = [loss(*[v + s * along if j == i else v for j, v in enumerate(at)]) for s in (step, -step)]
        slope_of = float((ends[0] - ends[1]) / (2 * step))
        terms = got[i].double() * along
        assert abs(slope_of - float(terms.sum())) <= ((n + D + F) * STEP + 1e-6) * float(terms.abs().sum()) + 1e-6


# ---- as programs call it ---------------------------------------------------------------------------------------------------
def test_same_bits_again_whatever_the_workspace_holds():
    n, D, F, t = 1111, 256, 1000, torch.bfloat16
    gen, x, wg, wu, wd = model(n, D, F, t, 3)
    block = FeedForward(wg, wu, wd, max_rows=n, training=True)
    d = torch.randn(n, D, generator=gen, device=DEV).to(t)
    runs = []
    for fill in (0, 255):
        block.workspace.fill_(fill)
        out, saved = torch.empty_like(x), torch.empty(n, 2 * F, dtype=t, device=DEV)
        got = [torch.empty_like(v) for v in (x, wg, wu, wd)]
        block.forward(x, out, saved=saved)
        block.workspace.fill_(fill)
        block.backward(x, saved, d, *got)
        runs.append([out, saved] + got)
    for a, b in zip(*runs):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_rows_do_not_depend_on_their_neighbours():
    """A row that is not finite spoils no other row's output."""
    n, D, F = 200, 132, 260
    for t in TYPES:
        gen, x, wg, wu, wd = model(n, D, F, t, 4)
        block = FeedForward(wg, wu, wd, max_rows=n)
        out, bad = torch.empty_like(x), torch.empty_like(x)
        block.forward(x, out)
        y = x.clone()
        y[5], y[77, 3], y[199] = float("nan"), float("inf"), float("-inf")
        block.forward(y, bad)
        keep = [i for i in range(n) if i not in (5, 77, 199)]
        assert torch.equal(out[keep], bad[keep]) and bool(torch.isnan(bad[5]).all())


def test_rows_far_apart():
    """The largest stride: 2100 rows lie more than 4 GiB apart.  All of a call's rows side by side in one buffer."""
    n, D, F, t = 2100, 64, 68, torch.bfloat16
    gen, a, wg, wu, wd = exact_case(n, D, F, t, 0, 12)
    wide = torch.full((n, 1 << 20), -7.0, dtype=t, device=DEV)
    x, r, out, d, d_x = (wide[:, i * D:(i + 1) * D] for i in range(5))
    x.copy_(a)
    r.copy_(whole(n, D, t, gen, 0.5))
    d.copy_(whole(n, D, t, gen, 0.1))
    g, u, h, y = relu_reference(x, wg, wu, wd)
    block, saved = FeedForward(wg, wu, wd, max_rows=n, activation="relu", training=True), torch.empty(n, 2 * F, dtype=t, device=DEV)
    drop, m = Dropout(0.5, state(79, 8)), factors(0.5, 79, 8, n, D)
    block.forward(x, out, residual=r, dropout=drop, saved=saved)
    assert torch.equal(out, (y * m + r.double()).to(t)) and torch.equal(x, a)
    grads = [torch.empty_like(w) for w in (wg, wu, wd)]
    block.backward(x, saved, d, d_x, *grads, add=d, dropout=drop)
    e = d.double() * m
    b = e @ wd.double()
    dg, du = b * u * (g > 0), b * g.clamp(min=0)
    assert torch.equal(d_x, (dg @ wg.double() + du @ wu.double() + d.double()).to(t))
    for got, w in zip(grads, (dg.t() @ x.double(), du.t() @ x.double(), e.t() @ h)):
        assert torch.equal(got, w.to(t))
    drop.apply(x, d_x, residual=r)
    assert torch.equal(d_x, (x.double() * m + r.double()).to(t))
    assert bool((wide[:, 5 * D:] == -7.0).all())


def test_in_place():
    n, D, F, t = 70, 64, 128, torch.float16
    gen, x, wg, wu, wd = model(n, D, F, t, 5)
    block = FeedForward(wg, wu, wd, max_rows=n)
    out = torch.empty_like(x)
    block.forward(x, out, residual=x)
    for kind in ("x", "residual"):
        y, r = x.clone(), x.clone()
        block.forward(y, y if kind == "x" else r, residual=r)
        assert torch.equal(y if kind == "x" else r, out)
    y = x.clone()
    block.forward(y, y, residual=y)                      # the residual stream in place
    assert torch.equal(y, out)


def test_no_rows():
    gen, x, wg, wu, wd = model(5, 64, 128, torch.bfloat16, 6)
    block = FeedForward(wg, wu, wd, max_rows=5, training=True)
    none, saved = x[:0], torch.empty(0, 256, dtype=torch.bfloat16, device=DEV)
    block.forward(none, none.clone(), saved=saved)
    grads = [torch.full_like(w, 9.0) for w in (wg, wu, wd)]
    block.backward(none, saved, none, none.clone(), *grads, accumulate=True)
    assert all(bool((w == 9).all()) for w in grads)
    block.backward(none, saved, none, none.clone(), *grads)
    assert all(bool((w == 0).all()) for w in grads)


def test_streams_and_shared_workspace():
    """Two blocks of unlike sizes with one workspace, their calls in order on another stream than the one they were made on."""
    t, side = torch.bfloat16, torch.cuda.Stream()
    gen, x, wg, wu, wd = model(300, 128, 512, t, 7)
    _, _, wg2, wu2, wd2 = model(300, 128, 260, t, 8)
    big = FeedForward(wg, wu, wd, max_rows=300, training=True)
    small = FeedForward(wg2, wu2, wd2, max_rows=300, activation="gelu", workspace=big.workspace)
    a, b, c = (torch.empty_like(x) for _ in range(3))
    big.forward(x, a, residual=x)
    small.forward(a, b, residual=a)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    big.forward(x, c, residual=x, stream=side)
    small.forward(c, c, residual=c, stream=side)
    with torch.cuda.stream(side):
        d = c.clone()
    del big, small
    side.synchronize()
    assert torch.equal(d, b)


def test_a_training_step_in_a_graph():
    """Lookup's dropout, the block and its gradients, replayed with eager work between the replays: each draws the masks that the state
    says, and gives the bits that eager calls give."""
    n, D, F, p, t = 260, 128, 260, 0.2, torch.bfloat16
    gen, x, wg, wu, wd = model(n, D, F, t, 10)
    d = torch.randn(n, D, generator=gen, device=DEV).to(t)

    def buffers():
        return {"x": torch.zeros_like(x), "out": torch.zeros_like(x), "saved": torch.zeros(n, 2 * F, dtype=t, device=DEV),
                "d_x": torch.zeros_like(x), "grads": [torch.zeros_like(w) for w in (wg, wu, wd)]}

    def step(block, b, s):
        Dropout(p, s, 0).apply(x, b["x"])
        block.forward(b["x"], b["out"], residual=b["x"], dropout=Dropout(p, s, 1), saved=b["saved"])
        block.backward(b["x"], b["saved"], d, b["d_x"], *b["grads"], add=d, dropout=Dropout(p, s, 1))
        Dropout(p, s, 0).apply(b["d_x"], b["d_x"])
        s[1] += 2

    s, block = state(4, 100), FeedForward(wg, wu, wd, max_rows=n, training=True)
    b = buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(block, b, s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(block, b, s)
    eager = FeedForward(wg, wu, wd, max_rows=n, training=True)
    for i in range(4):
        want, own = buffers(), state(4, 102 + 2 * i)
        graph.replay()
        step(eager, want, own)
        torch.cuda.synchronize()
        assert torch.equal(s, own)
        for k in ("x", "out", "saved", "d_x"):
            assert torch.equal(b[k], want[k]), (i, k)
        assert all(torch.equal(v, w) for v, w in zip(b["grads"], want["grads"]))


def test_refusals():
    n, D, F, t = 20, 64, 128, torch.bfloat16
    gen, x, wg, wu, wd = model(n, D, F, t, 11)
    block = FeedForward(wg, wu, wd, max_rows=n)
    out, saved = torch.empty_like(x), torch.empty(n, 2 * F, dtype=t, device=DEV)

    def code(call):
        with pytest.raises(EcrmError) as e:
            call()
        return e.value.code

    more = torch.zeros(n + 1, D, dtype=t, device=DEV)
    assert code(lambda: block.forward(more, torch.empty_like(more))) == ECRM_EBATCH
    assert code(lambda: block.backward(x, saved, x, out)) == ECRM_ESCRATCH            # not made for training
    assert code(lambda: block.forward(more[1:], more[:n])) == ECRM_EINVAL             # rows apart by one
    assert code(lambda: block.forward(x, out, residual=more[1:], saved=None, dropout=Dropout(2.0, state()))) == ECRM_EINVAL
    assert code(lambda: block.forward(x, wd[:n, :D])) == ECRM_EINVAL                  # a weight
    own = block.workspace[:n * D * 2].view(t).view(n, D)
    assert code(lambda: block.forward(x, own)) == ECRM_EINVAL
    assert code(lambda: block.forward(own, out)) == ECRM_EINVAL
    assert code(lambda: block.forward(x, out, residual=own)) == ECRM_EINVAL
    assert code(lambda: block.forward(x[:4], out[:4], saved=x.flatten()[:4 * 2 * F].view(4, 2 * F))) == ECRM_EINVAL
    with pytest.raises(EcrmError):
        FeedForward(wg, wu, wd, max_rows=n, workspace=torch.empty(1024, dtype=torch.uint8, device=DEV))
    with pytest.raises(AssertionError):
        block.forward(x.float(), out)
    with pytest.raises(AssertionError):
        block.forward(x, out, saved=saved[:, :F])
    with pytest.raises(AssertionError):
        FeedForward(wg, wu, wd.t(), max_rows=n)
    train = FeedForward(wg, wu, wd, max_rows=n, training=True)
    grads = [torch.empty_like(w) for w in (wg, wu, wd)]
    assert code(lambda: train.backward(x, saved, x, out, grads[0], None, grads[2])) == ECRM_EINVAL
    assert code(lambda: train.backward(x, saved, x, out, grads[0], grads[0], grads[2])) == ECRM_EINVAL
    assert code(lambda: train.backward(x, saved, x, out, wg, grads[1], grads[2])) == ECRM_EINVAL
    d = x.clone()
    assert code(lambda: train.backward(x, saved, d, x)) == ECRM_EINVAL                # the place of x
    assert code(lambda: train.backward(x, saved, d, saved[:, :D])) == ECRM_EINVAL
    train.backward(x, saved, d)                                                       # nothing is wanted


def test_the_mask_state_lies_outside_the_workspace():
    n, D, F, t = 20, 64, 128, torch.bfloat16
    gen, x, wg, wu, wd = model(n, D, F, t, 12)
    block = FeedForward(wg, wu, wd, max_rows=n, training=True)
    out, saved = torch.empty_like(x), torch.empty(n, 2 * F, dtype=t, device=DEV)
    words = block.workspace[:256].view(torch.int64)
    for inside in (words[:2], words[16:18]):
        with pytest.raises(EcrmError) as e:
            block.forward(x, out, dropout=Dropout(0.5, inside), saved=saved)
        assert e.value.code == ECRM_EINVAL
        with pytest.raises(EcrmError) as e:
            block.backward(x, saved, x, out, dropout=Dropout(0.5, inside))
        assert e.value.code == ECRM_EINVAL


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The block, or the mask, taken for one of device 1."""
    n, D, F, t = 4, 64, 128, torch.bfloat16
    gen, x, wg, wu, wd = model(n, D, F, t, 13)
    out, saved = torch.empty_like(x), torch.empty(n, 2 * F, dtype=t, device=DEV)
    block, drop = FeedForward(wg, wu, wd, max_rows=n, training=True), Dropout(0.5, state())
    drop._device = 1
    for call in (lambda: block.forward(x, out, dropout=drop), lambda: block.backward(x, saved, x, out, dropout=drop), lambda: drop.apply(x, out)):
        with pytest.raises(AssertionError):
            call()
    block._device = 1
    for call in (lambda: block.forward(x, out), lambda: block.backward(x, saved, x, out)):
        with pytest.raises(AssertionError):
            call()
    block._device = 0
    for call in (lambda: block.forward(x.cpu(), out), lambda: block.forward(x, out.cpu()), lambda: FeedForward(wg, wu.cpu(), wd, max_rows=n)):
        with pytest.raises(AssertionError):
            call()
    monkeypatch.setattr("paper_2104_01981_amd.binding._raw_device", lambda: 1)
    for call in (lambda: block.forward(x, out), lambda: Dropout(0.5, state()).apply(x, out)):
        with pytest.raises(AssertionError):
            call()
