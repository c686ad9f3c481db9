"""Dropout whose masks are never stored (ecrm_dropout, ecrm_embed_dropout, ecrm_embed_grad_dropout, ecrm_embed_grad_dense_dropout): the
masks bit for bit, sizes that end inside a block of eight columns, strides, in place, values that are not finite, all types.

Tolerances are roundings: half a step of a type is eps / 2 relative to the value.  The factor is rounded to 32 bits, its product with the
element, the sum with the residual; then comes the rounding to the type.  Sums of a gradient are formed in 64 bits and rounded once."""
import numpy as np
import pytest
import torch

import philox
import synth_inputs as si
from paper_2104_01981_amd import Dropout, Ecrm, EcrmError

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}    # smallest steps
PAD = -100


def half(t):
    return torch.finfo(t).eps / 2


def state(seed=0x123456789ABCDEF0, number=7):
    words = np.array([seed % (1 << 64), number % (1 << 64)], dtype=np.uint64).view(np.int64)
    return torch.from_numpy(words).to(DEV)


def factors(p, seed, number, rows, cols, first_row=0):
    return torch.from_numpy(philox.kept(p, seed, number, rows, cols, first_row) * philox.factor(p)).to(DEV)


def values(n, D, t, seed, extra=0, fill=float("nan")):
    g = torch.Generator(device=DEV).manual_seed(seed)
    wide = torch.full((n + 1, D + extra), fill, dtype=t, device=DEV)
    wide[:n, extra:] = torch.randn(n, D, generator=g, device=DEV).to(t)
    return wide[:n, extra:], wide                        # from a multiple of four elements on, not always of 16 bytes


# ---- by itself -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,D,extra", [(1, 4, 0), (1, 8, 4), (2, 12, 0), (3, 16, 8), (63, 20, 4), (65, 128, 0), (100, 132, 12), (700, 64, 0),
                                       (1025, 100, 4), (4097, 260, 0), (5, 65536, 0), (3000, 512, 8)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(t, n, D, extra, residual):
    p, seed, number, offset = 0.3, -3 + n, (1 << 32) - 5, 4 + D
    x, _ = values(n, D, t, n + D, extra)
    r = values(n, D, t, n * D, 2 * extra)[0] if residual else None
    out, around = values(n, D, t, 1, extra, fill=-7.0)
    drop = Dropout(p, state(seed, number), offset)
    drop.apply(x, out, residual=r)
    y = x.double() * factors(p, seed, number + offset, n, D)
    want = y + r.double() if residual else y
    tol = (half(t) + 2.0 ** -24) * (1 + 2.0 ** -20) * want.abs() + 2 * 2.0 ** -24 * (1 + 2.0 ** -20) * y.abs() + TINY[t]
    assert bool(((out.double() - want).abs() <= tol).all())
    if not residual:                                    # the mask, bit for bit
        assert torch.equal(out == 0, (y == 0) | (x == 0))
    assert bool((around[n] == -7.0).all()) and bool((around[:, :extra] == -7.0).all())
    for into in [x] + ([r] if residual else []):         # in place
        keep = out.clone()
        drop.apply(x, into, residual=r)
        assert torch.equal(into, keep)
        x = values(n, D, t, n + D, extra)[0]


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -17, 1.0 / 65536, 0.1, 0.999, 1.0 - 2.0 ** -18, 1.0])
def test_probabilities(p):
    n, D = 257, 516
    x, _ = values(n, D, torch.float32, 5)
    out = torch.empty_like(x)
    Dropout(p, state(11, 12), 1).apply(x, out)
    want = x.double() * factors(p, 11, 13, n, D)
    assert bool(((out.double() - want).abs() <= 2 * 2.0 ** -24 * (1 + 2.0 ** -20) * want.abs()).all())
    assert torch.equal(out == 0, want == 0)


def test_what_is_dropped_is_zero_whatever_it_was():
    n, D, p = 64, 128, 0.5
    for t in TYPES:
        x = torch.full((n, D), float("nan"), dtype=t, device=DEV)
        x[1::2] = float("inf")
        out, r = torch.empty_like(x), torch.ones_like(x)
        Dropout(p, state()).apply(x, out, residual=r)
        m = factors(p, 0x123456789ABCDEF0, 7, n, D) > 0
        assert bool((out[~m] == 1).all())
        assert bool(torch.isnan(out[0::2][m[0::2]]).all()) and bool(torch.isinf(out[1::2][m[1::2]]).all())


def test_masks_differ_by_number_and_offset_and_agree():
    n, D = 100, 256
    x = torch.ones(n, D, device=DEV)
    s = state(5, 100)

    def drawn(drop):
        out = torch.empty_like(x)
        drop.apply(x, out)
        return out

    a, b, again = drawn(Dropout(0.5, s, 0)), drawn(Dropout(0.5, s, 1)), drawn(Dropout(0.5, s, 0))
    assert torch.equal(a, again)
    # independent masks of 25600 elements agree in half of them: five standard deviations
    assert abs(float(((a == 0) == (b == 0)).double().mean()) - 0.5) < 5 * 0.5 / (n * D) ** 0.5
    s[1] += 1
    assert torch.equal(drawn(Dropout(0.5, s, 0)), b) and torch.equal(drawn(Dropout(0.5, s, -1)), a)


def test_rows_beyond_what_a_launch_has():
    """A launch has at most 2^30 blocks of eight columns: more rows than that in one of 2^24 columns."""
    n, D, p = 513, 1 << 24, 0.25
    free, _ = torch.cuda.mem_get_info()
    if free < 3 * n * D * 2:
        pytest.skip("not enough device memory")
    x = torch.ones(n, D, dtype=torch.bfloat16, device=DEV)
    Dropout(p, state(3, 4)).apply(x, x)
    for row, at in ((0, 0), (511, D - 1024), (512, 0), (512, D - 1024)):
        # of a block of 1024 columns: the same masks with the blocks' numbers, row by row
        blocks = np.arange(at // 8, at // 8 + 128, dtype=np.uint64)
        w = philox.philox([blocks, np.uint64(row) + 0 * blocks, np.uint64(4) + 0 * blocks, 0 * blocks], (3, 0))
        bits = np.stack([h for q in w for h in (q & np.uint64(0xFFFF), q >> np.uint64(16))], -1).reshape(-1)
        assert np.array_equal((x[row, at:at + 1024] != 0).cpu().numpy(), bits >= philox.border(p))


def test_dropout_in_a_graph_draws_what_the_state_says():
    n, D, p = 300, 132, 0.4
    x, _ = values(n, D, torch.bfloat16, 1)
    out, s = torch.zeros_like(x), state(9, 50)
    drop = Dropout(p, s, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        drop.apply(x, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        drop.apply(x, out)
        s[1] += 3
    for step in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(x)
        Dropout(p, state(9, 50 + 3 * step), 2).apply(x, eager)
        assert torch.equal(out, eager) and int(s[1]) == 50 + 3 * (step + 1)


def test_python_refuses():
    x = torch.zeros(4, 16, device=DEV)
    with pytest.raises(AssertionError):
        Dropout(0.5, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(AssertionError):
        Dropout(0.5, state()[:1])
    drop = Dropout(0.5, state())
    with pytest.raises(AssertionError):
        drop.apply(x, torch.zeros(4, 16, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(AssertionError):
        drop.apply(x, x.t())
    with pytest.raises(EcrmError):
        Dropout(2.0, state()).apply(x, x)
    with pytest.raises(EcrmError):
        drop.apply(x[1:], x[:3])                         # rows apart by one: neither in place nor clear
    drop.apply(x[:0], x[:0])


def test_interleaved_columns_are_apart():
    wide = torch.zeros(9, 64, device=DEV)
    wide[:, :32] = 1.0
    Dropout(0.5, state(1, 1)).apply(wide[:, :32], wide[:, 32:])
    assert bool((wide[:, :32] == 1).all())
    assert torch.equal(wide[:, 32:], factors(0.5, 1, 1, 9, 32).float())


# ---- lookup and its gradient -----------------------------------------------------------------------------------------------
class Table:
    def __init__(self, R, D, k=4, S=5, max_batch=1 << 16, seed=3):
        self.R, self.D, self.k = R, D, k
        self.E = si.table(seed, si.TAG_E0, R, D, DEV)
        self.A = si.table(seed, si.TAG_A0, R, D, DEV)
        self.PE, self.PA = torch.zeros(R // k, D, device=DEV), torch.zeros(R // k, D, device=DEV)
        self.load = torch.zeros(2, S, dtype=torch.int64, device=DEV)
        self.ctx = Ecrm(R, D, k, S, max_batch=max_batch)
        self.scratch = torch.full((self.ctx.scratch_bytes(),), 0xA5, dtype=torch.uint8, device=DEV)
        self.ctx.bind(self.E, self.A, self.PE, self.PA, self.load[0], self.load[1], self.scratch)
        self.ctx.encode()


def tokens(R, n, kind, seed, padding=0.1):
    rng = np.random.default_rng(seed)
    if kind == "uniform":
        t = rng.integers(0, R, n)
    elif kind == "text":
        t = np.minimum(np.power(R + 1.0, rng.random(n)).astype(np.int64) - 1, R - 1)
    else:
        t = np.full(n, R - 1)
    return torch.from_numpy(np.where(rng.random(n) < padding, PAD, t).astype(np.int64)).to(DEV)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,k,S", [(4, 1, 2), (8, 4, 5), (12, 3, 4), (36, 2, 3), (128, 4, 5), (132, 2, 5), (1024, 4, 5)])
def test_lookup_with_dropout(D, k, S, t):
    R, n, p, scale = 250 * k, 1003, 0.2, float(np.float32(D ** 0.5))
    tab = Table(R, D, k, S, max_batch=8)
    keys = tokens(R, n, "uniform", D)
    drop = Dropout(p, state(D, 1 << 40), 3)
    m = factors(p, D, (1 << 40) + 3, n, D)
    plain = torch.where((keys != PAD)[:, None], tab.E.double()[keys.clamp(min=0)] * scale, torch.zeros((), dtype=torch.float64, device=DEV))
    for lost in (None, S - 1):
        for rows, extra in ((1, 0), (63, 4), (64, 0), (n, 12)):
            out, around = values(rows, D, t, 1, extra, fill=-7.0)
            tab.ctx.embed(keys[:rows], out, scale=scale, padding=PAD, lost_server=lost, dropout=drop)
            want = plain[:rows] * m[:rows]
            # product with the scale, factor, product with the factor; a decoded entry is off by a rounding of a sum of k + 1 of size <= 1
            tol = (half(t) + 3 * 2.0 ** -24) * (1 + 2.0 ** -20) * want.abs() + TINY[t]
            if lost is not None:
                tol = tol + scale * philox.factor(p) * (k + 2) * 2.0 ** -24
            assert bool(((out.double() - want).abs() <= tol).all())
            if lost is None:
                assert torch.equal(out == 0, want.to(t) == 0)
            assert bool((around[rows] == -7.0).all()) and bool((around[:, :extra] == -7.0).all())
    assert tab.ctx.status() == 0


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,n,kind", [(4, 1, "uniform"), (8, 64, "text"), (12, 255, "one"), (36, 256, "uniform"), (128, 257, "text"),
                                      (128, 1536, "text"), (132, 1537, "one"), (128, 8193, "text"), (20, 5000, "one"), (256, 20000, "uniform"),
                                      (1024, 600, "text"), (1024, 3000, "text"), (128, 70001, "text")])
def test_gradient_with_dropout(D, n, kind, t):
    R, p, scale = 4 * 500, 0.3, float(np.float32(D ** 0.5))
    tab = Table(R, D, max_batch=n)
    keys = tokens(R, n, kind, n)
    keys[0] = 5
    d, _ = values(n, D, t, n, extra=4)
    drop = Dropout(p, state(n, -1), 0)
    m = factors(p, n, -1, n, D)
    d[(m == 0)] = float("nan")                           # what was dropped counts for nothing
    d[keys == PAD] = float("inf")
    terms = torch.where(m > 0, d.double(), torch.zeros((), dtype=torch.float64, device=DEV)) * m
    at = (keys != PAD).nonzero().flatten()
    names, where = torch.unique(keys[at], return_inverse=True)
    sums = torch.zeros(len(names), D, dtype=torch.float64, device=DEV).index_add(0, where, terms[at]) * scale
    mags = torch.zeros(len(names), D, dtype=torch.float64, device=DEV).index_add(0, where, terms[at].abs()) * scale
    out_keys = torch.full((n,), 77, dtype=torch.int64, device=DEV)
    grads = torch.full((n, D), 77.0, device=DEV)
    count = torch.zeros(1, dtype=torch.int64, device=DEV)
    tab.ctx.embed_grad(keys, d, out_keys, grads, count, scale=scale, padding=PAD, dropout=drop)
    u = int(count)
    assert torch.equal(out_keys[:u], names) and bool((out_keys[u:] == -1).all()) and bool((grads[u:] == 77.0).all())
    tol = half(torch.float32) * sums.abs() + 2 * (n + 4) * 2.0 ** -53 * mags + TINY[torch.float32]
    assert bool(((grads[:u].double() - sums).abs() <= tol).all())
    dense = torch.full((R, D), 3.0, device=DEV)
    tab.ctx.embed_grad_dense(keys, d, dense, scale=scale, padding=PAD, dropout=drop)
    want = torch.zeros(R, D, dtype=torch.float64, device=DEV)
    want[names] = sums
    assert bool(((dense[names].double() - sums).abs() <= tol).all())
    assert int((dense != 0).any(1).sum()) <= len(names)
    more = dense.clone()
    tab.ctx.embed_grad_dense(keys, d, more, scale=scale, padding=PAD, accumulate=True, dropout=drop)
    tol2 = half(torch.float32) * (sums + dense[names].double()).abs() + 2 * (n + 4) * 2.0 ** -53 * mags + TINY[torch.float32]
    assert bool(((more[names].double() - dense[names].double() - sums).abs() <= tol2).all())
    assert tab.ctx.status() == 0


def test_rows_past_the_caches():
    """A batch that is moved past the caches, and read ahead beside the sort."""
    R, D, n, p = 4 * 50000, 128, 1 << 18, 0.1
    tab = Table(R, D, max_batch=n)
    keys = tokens(R, n, "uniform", 1)
    d, _ = values(n, D, torch.float32, 2)
    m = factors(p, 21, 22, n, D)
    out_keys, grads = torch.empty(n, dtype=torch.int64, device=DEV), torch.empty(n, D, device=DEV)
    count = torch.zeros(1, dtype=torch.int64, device=DEV)
    tab.ctx.embed_grad(keys, d, out_keys, grads, count, padding=PAD, dropout=Dropout(p, state(21, 22)))
    at = (keys != PAD).nonzero().flatten()
    names, where = torch.unique(keys[at], return_inverse=True)
    terms = d[at].double() * m[at]
    sums = torch.zeros(len(names), D, dtype=torch.float64, device=DEV).index_add(0, where, terms)
    mags = torch.zeros(len(names), D, dtype=torch.float64, device=DEV).index_add(0, where, terms.abs())
    u = int(count)
    assert torch.equal(out_keys[:u], names)
    assert bool(((grads[:u].double() - sums).abs() <= half(torch.float32) * sums.abs() + 2 * 40 * 2.0 ** -53 * mags + TINY[torch.float32]).all())


def test_lookup_with_dropout_refuses():
    tab = Table(1024, 64, max_batch=100)
    keys, out = tokens(1024, 50, "uniform", 1), torch.zeros(50, 64, device=DEV)
    for drop in (Dropout(-0.5, state()), Dropout(1.5, state()), Dropout(float("nan"), state())):
        with pytest.raises(EcrmError):
            tab.ctx.embed(keys, out, padding=PAD, dropout=drop)
        with pytest.raises(EcrmError):
            tab.ctx.embed_grad_dense(keys, out, torch.zeros(1024, 64, device=DEV), padding=PAD, dropout=drop)
    whole = torch.zeros(50 * 64 + 4, device=DEV)
    inside = Dropout(0.5, whole[8:12].view(torch.int64))
    with pytest.raises(EcrmError):
        tab.ctx.embed(keys, whole[:50 * 64].view(50, 64), padding=PAD, dropout=inside)
    with pytest.raises(EcrmError):
        tab.ctx.embed_grad(keys, out, torch.zeros(50, dtype=torch.int64, device=DEV), whole[:50 * 64].view(50, 64),
                           torch.zeros(1, dtype=torch.int64, device=DEV), padding=PAD, dropout=inside)
