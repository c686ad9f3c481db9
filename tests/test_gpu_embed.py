"""Looking tokens up and the gradient by sorted tokens (ecrm_embed, ecrm_embed_grad, ecrm_embed_grad_dense) against plain
64-bit forms, where they can go wrong: rows of any width, numbers of tokens around what a lane, a team and a workgroup take, one
token many times beside others once, padding, padding alone, types, strides, tokens out of range, values that are not finite.

Tolerances are roundings: half a step of a type is eps / 2 relative to the value.  The lookup rounds a product to 32 bits and
then to its type; a gradient is summed in 64 bits and rounded once to 32."""
import numpy as np
import pytest
import torch

import oracle
import synth_inputs as si
from paper_2104_01981_amd import ECRM_EBATCH, ECRM_EINVAL, ECRM_EKEYRANGE, ECRM_ESCRATCH, Ecrm, EcrmError

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
PAD = -100
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}    # smallest steps


def half(t):
    return torch.finfo(t).eps / 2


class Table:
    def __init__(self, R, D, k=4, S=5, max_batch=1 << 16, seed=3):
        self.R, self.D, self.k, self.S = R, D, k, S
        self.E = si.table(seed, si.TAG_E0, R, D, DEV)
        self.A = si.table(seed, si.TAG_A0, R, D, DEV)
        self.PE, self.PA = torch.zeros(R // k, D, device=DEV), torch.zeros(R // k, D, device=DEV)
        self.load = torch.zeros(2, S, dtype=torch.int64, device=DEV)
        self.ctx = Ecrm(R, D, k, S, max_batch=max_batch)
        size = self.ctx.scratch_bytes()
        self.scratch = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device=DEV)       # whatever lies in it
        self.behind = self.scratch[size:]
        self.ctx.bind(self.E, self.A, self.PE, self.PA, self.load[0], self.load[1], self.scratch[:size])
        self.ctx.encode()


def tokens(R, n, kind, seed, padding=0.0):
    """n tokens: uniform; `text`: a few of them are most of the batch; `one`: all the same; `runs`: two, in long runs, and others."""
    rng = np.random.default_rng(seed)
    if kind == "uniform":
        t = rng.integers(0, R, n)
    elif kind == "text":
        t = np.minimum(np.power(R + 1.0, rng.random(n)).astype(np.int64) - 1, R - 1)
    elif kind == "one":
        t = np.full(n, R - 1)
    else:
        t = rng.choice(np.array([0, R - 1, R // 2]), n)
        t[::7] = rng.integers(0, R, len(t[::7]))
    if padding:
        t = np.where(rng.random(n) < padding, PAD, t)
    return torch.from_numpy(t.astype(np.int64)).to(DEV)


def gradients(n, D, t, seed, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    wide = torch.full((n, D + extra), float("nan"), dtype=t, device=DEV)
    wide[:, :D] = torch.randn(n, D, generator=g, device=DEV).to(t)
    return wide[:, :D]


def reference(keys, d, scale, padding):
    """Distinct tokens and, in 64 bits, their sums and the sums of the absolute values."""
    real = (keys != padding).nonzero().flatten() if padding is not None else torch.arange(len(keys), device=DEV)
    names, where = torch.unique(keys[real], return_inverse=True)
    x = d[real].double()
    # of a few rows, several places each, so that not all of a token's terms meet in one
    ways = max(1, min(64, (1 << 23) // max(1, len(names) * d.shape[1])))
    where = where * ways + torch.arange(len(where), device=DEV) % ways
    parts = torch.zeros(len(names) * ways, d.shape[1], dtype=torch.float64, device=DEV)
    sums = parts.index_add(0, where, x).view(len(names), ways, -1).sum(1)
    mags = parts.index_add(0, where, x.abs()).view(len(names), ways, -1).sum(1)
    return names, sums * scale, mags * abs(scale)


def close(got, want, mags, n, t=torch.float32):
    """One rounding of the result; 64-bit sums of at most n terms, in any order, on both sides."""
    tol = half(t) * want.abs() + 2 * (n + 2) * 2.0 ** -53 * mags + TINY[t]
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()}, at most {float((got.double() - want).abs().max())}"


def run_grad(tab, keys, d, scale=1.0, padding=PAD, room=3, **kw):
    n = len(keys)
    ok = torch.full((n + room,), 77, dtype=torch.int64, device=DEV)
    og = torch.full((n + room, tab.D), 77.0, device=DEV)
    count = torch.full((1,), 77, dtype=torch.int64, device=DEV)
    tab.ctx.embed_grad(keys, d, ok, og, count, scale=scale, padding=padding, **kw)
    u = int(count)
    assert bool((ok[n:] == 77).all()) and bool((ok[u:n] == -1).all()) and bool((og[u:] == 77.0).all())
    return ok[:u], og[:u]


def check_grad(tab, keys, d, scale=1.0, padding=PAD):
    names, sums, mags = reference(keys, d, scale, padding)
    ok, og = run_grad(tab, keys, d, scale, padding)
    assert torch.equal(ok, names)
    close(og, sums, mags, len(keys))
    again = run_grad(tab, keys, d, scale, padding)
    assert torch.equal(again[0], ok) and torch.equal(again[1].view(torch.int32), og.view(torch.int32))
    return names, sums, mags


# ---- lookup ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,k,S", [(4, 1, 2), (12, 3, 4), (36, 2, 3), (128, 4, 5), (260, 10, 11), (1024, 2, 5)])
@pytest.mark.parametrize("t", TYPES)
def test_lookup(D, k, S, t):
    R, scale, n = k * 333, float(np.float32(D ** 0.5)), 4099
    tab = Table(R, D, k, S, max_batch=8)
    keys = tokens(R, n, "uniform", D, padding=0.1)
    want = torch.where((keys != PAD)[:, None], tab.E.double()[keys.clamp(min=0)] * scale, torch.zeros((), dtype=torch.float64, device=DEV))
    for m, extra in ((1, 0), (2, 4), (63, 0), (64, 8), (65, 0), (1000, 4), (n, 0), (n, 12)):
        wide = torch.full((m + 1, D + extra), -7.0, dtype=t, device=DEV)
        tab.ctx.embed(keys[:m], wide[:m, :D], scale=scale, padding=PAD)
        got, ref = wide[:m, :D].double(), want[:m]
        assert bool(((got - ref).abs() <= (half(t) + 2.0 ** -24) * (1 + 2.0 ** -20) * ref.abs() + TINY[t]).all())
        assert bool((wide[m] == -7.0).all()) and bool((wide[:, D:] == -7.0).all())
    assert tab.ctx.status() == 0


@pytest.mark.parametrize("D,k,S", [(4, 1, 2), (36, 3, 4), (128, 4, 5), (132, 10, 11), (512, 2, 7)])
def test_lookup_while_a_server_is_down(D, k, S):
    """The decoded entries are those of a degraded read; in 32 bits and with a scale of one the same bits."""
    R, n, lost = k * 500, 5003, S - 1
    tab = Table(R, D, k, S, max_batch=8)
    tab.ctx.fail_server(lost)
    keys = tokens(R, n, "uniform", D, padding=0.05)
    found = keys != PAD
    read = torch.zeros(n, D, device=DEV)
    tab.ctx.degraded_read(keys.clamp(min=0), lost, read)
    read[~found] = 0.0
    hE, hA, hPE, hPA = (x.cpu().numpy() for x in (tab.E, tab.A, tab.PE, tab.PA))
    he, _ = oracle.degraded_read(hE, hA, hPE, hPA, k, S, keys.clamp(min=0).cpu().numpy().astype(np.uint64), lost)
    assert np.array_equal(read[found].cpu().numpy(), he[found.cpu().numpy()])
    for t, scale in ((torch.float32, 1.0), (torch.bfloat16, 0.5), (torch.float16, 3.0)):
        out = torch.full((n, D), float("nan"), dtype=t, device=DEV)
        tab.ctx.embed(keys, out, scale=scale, padding=PAD, lost_server=lost)
        assert torch.equal(out, (read * scale).to(t))
    assert tab.ctx.status() == 0


def test_lookup_of_values_at_the_ends_of_the_types():
    tab = Table(64, 4, max_batch=8)
    v = torch.tensor([[float("inf"), float("-inf"), float("nan"), -0.0], [65504.0, 65520.0, 3.0e38, 3.4e38],
                      [1e-40, -1e-45, 2.0 ** -24, 2.0 ** -25], [1.0 + 2.0 ** -8, 1.0 + 3 * 2.0 ** -8, 2.0 ** -133, 2.0 ** -134]])
    tab.E[:4] = v.to(DEV)
    keys = torch.tensor([0, 1, 2, 3], device=DEV)
    for t in TYPES:
        out = torch.empty(4, 4, dtype=t, device=DEV)
        tab.ctx.embed(keys, out)
        torch.testing.assert_close(out.cpu(), v.to(t), rtol=0, atol=0, equal_nan=True)


def test_lookup_leaves_rows_of_bad_tokens_and_says_so():
    tab = Table(1 << 10, 36, max_batch=8)
    keys = tokens(1 << 10, 300, "uniform", 1, padding=0.2)
    bad = keys.clone()
    bad[17], bad[255], bad[299] = 1 << 10, -1, 1 << 40
    good, out = torch.empty(300, 36, device=DEV), torch.full((300, 36), 5.0, device=DEV)
    tab.ctx.embed(keys, good, padding=PAD)
    assert tab.ctx.status() == 0
    tab.ctx.embed(bad, out, padding=PAD)
    assert tab.ctx.status() == ECRM_EKEYRANGE
    tab.ctx.clear_status()
    hit = torch.zeros(300, dtype=torch.bool, device=DEV)
    hit[[17, 255, 299]] = True
    assert bool((out[hit] == 5.0).all()) and torch.equal(out[~hit], good[~hit])
    tab.ctx.embed(keys, out)                              # the padding token is a bad one where there is no padding
    assert tab.ctx.status() == ECRM_EKEYRANGE
    tab.ctx.clear_status()
    for pad in (7, -1, 1 << 10):                          # a row as well; the key behind the last one; just no row
        there = torch.where(keys <= 7, torch.full_like(keys, pad), keys)
        tab.ctx.embed(there, out, padding=pad)
        assert tab.ctx.status() == 0 and bool((out[keys <= 7] == 0).all()) and torch.equal(out[keys > 7], good[keys > 7])
        check_grad(tab, there[:8], out[:8], padding=pad)
        assert tab.ctx.status() == 0


# ---- gradient --------------------------------------------------------------------------------------------------------------
SIZES = [1, 2, 3, 5, 31, 64, 100, 255, 256, 257, 1023, 1024, 1025, 4097, 8192, 8193]


@pytest.mark.parametrize("D", [4, 12, 36, 128, 252, 512, 1020, 1024])
@pytest.mark.parametrize("kind", ["uniform", "text", "one", "runs"])
def test_gradient(D, kind):
    R = 4 * 301
    tab = Table(R, D)
    for i, n in enumerate(SIZES):
        t = TYPES[i % 3]
        keys = tokens(R, n, kind, 10 + i, padding=0.15 if i % 2 else 0.0)
        check_grad(tab, keys, gradients(n, D, t, i, extra=(0, 4, 20)[i % 3]), scale=float(np.float32((1.0, -0.3, D ** 0.5)[i % 3])))
    assert tab.ctx.status() == 0


@pytest.mark.parametrize("R,D,n,kind", [(1 << 10, 128, 70001, "text"), (1 << 20, 128, 65535, "text"), (1 << 17, 16, 40961, "runs"), (1 << 32 >> 6, 4, 30000, "text"), (1 << 20, 128, 70001, "text"), (1 << 20, 64, 70001, "uniform"),
                                        (1 << 22, 4, 300007, "text"), (1 << 12, 256, 100003, "one"), (4, 32, 50000, "uniform"),
                                        (1 << 16, 16, 600011, "runs"), (1 << 24, 8, 600011, "text"), (1 << 14, 1024, 20011, "text"), (1 << 11, 32, 65536, "text"), (1 << 12, 32, 65537, "uniform"),
                                        (1 << 20, 12, 262144, "runs"), (1 << 26, 4, 262145, "text"), ((1 << 22) + 4, 4, 2100003, "uniform"),
                                        (1 << 9, 4, 5000011, "text"), (1 << 22, 8, 100003, "text"), ((1 << 22) - 4, 16, 262143, "uniform")])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_gradient_of_larger_batches(R, D, n, kind, t):
    tab = Table(R, D, max_batch=n)
    check_grad(tab, tokens(R, n, kind, n, padding=0.07), gradients(n, D, t, 5), scale=float(np.float32(D ** 0.5)))
    assert tab.ctx.status() == 0


@pytest.mark.parametrize("R,D,n,t,extra", [(1 << 14, 1024, 18001, torch.bfloat16, 8), (1 << 14, 1020, 18001, torch.float16, 0),
                                           (1 << 12, 512, 27011, torch.float32, 4), (1 << 16, 256, 70001, torch.float16, 4),
                                           (1 << 12, 36, 900001, torch.float32, 12), (1 << 18, 128, 300007, torch.bfloat16, 64)])
def test_gradient_of_rows_past_the_caches(R, D, n, t, extra):
    """Rows of more than 100 MiB together, some of which are read ahead: 16 bytes at a time where all of them are so aligned."""
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, "text", n, padding=0.05), gradients(n, D, t, 7, extra=extra)
    names, sums, mags = check_grad(tab, keys, d)
    old = torch.randn(R, D, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    dE = old.clone()
    tab.ctx.embed_grad_dense(keys, d, dE, padding=PAD, accumulate=True)
    close(dE[names], sums + old[names].double(), mags + old[names].double().abs(), n)
    away = torch.isin(torch.arange(R, device=DEV), names, invert=True)
    assert torch.equal(dE[away], old[away]) and tab.ctx.status() == 0


@pytest.mark.parametrize("D", [4, 128, 296, 1024])
def test_scratch_of_exactly_the_batch(D):
    """Contexts whose scratch buffer serves this batch and no larger one, at the sizes where the way changes."""
    for n in (1, 256, 257, 1536, 1537, 8192, 8193, 65536, 65537, 262144, 262145):
        if n * D > 1 << 26:
            continue
        for R in (1 << 11, (1 << 11) + 4, 1 << 21):
            tab = Table(R, D if R < 1 << 20 or D <= 128 else 64, max_batch=n)
            check_grad(tab, tokens(R, n, "text", n, padding=0.1), gradients(n, tab.D, torch.bfloat16, 1))
            dE = torch.full((R, tab.D), 3.0, device=DEV)
            tab.ctx.embed_grad_dense(tokens(R, n, "runs", n), gradients(n, tab.D, torch.float32, 2), dE)
            assert bool((tab.behind == 0xA5).all()) and tab.ctx.status() == 0


@pytest.mark.parametrize("n", [1, 100, 1000, 5000, 20000, 66000])
def test_gradient_of_padding_alone(n):
    tab = Table(1 << 10, 36, max_batch=n)
    keys = torch.full((n,), PAD, dtype=torch.int64, device=DEV)
    names, grads = run_grad(tab, keys, torch.full((n, 36), float("nan"), device=DEV))
    assert len(names) == 0 and len(grads) == 0
    dE = torch.full((1 << 10, 36), 3.0, device=DEV)
    tab.ctx.embed_grad_dense(keys, torch.full((n, 36), float("nan"), device=DEV), dE, padding=PAD, accumulate=True)
    assert bool((dE == 3.0).all())
    tab.ctx.embed_grad_dense(keys, torch.full((n, 36), float("nan"), device=DEV), dE, padding=PAD)
    assert bool((dE == 0.0).all()) and tab.ctx.status() == 0


@pytest.mark.parametrize("n", [40, 1000, 3000, 40000, 90000])
def test_values_that_are_not_finite_stay_in_their_row(n):
    """... whether their run lies in one chunk or goes over many, and in padded places they do not count."""
    R, D = 1 << 10, 36
    tab = Table(R, D, max_batch=n)
    keys = tokens(R, n, "text", n, padding=0.1)
    d = gradients(n, D, torch.bfloat16, 3).contiguous()
    d[keys == PAD] = float("nan")
    hot, other = keys[keys != PAD].mode().values, keys[keys != PAD].max()
    d[(keys == hot).nonzero()[0], 5] = float("inf")
    d[(keys == other).nonzero()[-1], 7] = float("nan")
    names, grads = run_grad(tab, keys, d)
    ref, sums, mags = reference(keys, d, 1.0, PAD)
    assert torch.equal(names, ref)
    fine = torch.isfinite(sums)
    assert int((~fine).sum()) == 2 and torch.equal(torch.isnan(grads), torch.isnan(sums)) and torch.equal(torch.isinf(grads), torch.isinf(sums))
    close(grads[fine], sums[fine], mags[fine], n)


@pytest.mark.parametrize("R,D,n", [(1 << 10, 36, 1), (1 << 10, 36, 3000), (1 << 14, 128, 20011), (1 << 10, 256, 70001)])
@pytest.mark.parametrize("kind", ["uniform", "text"])
def test_dense_gradient(R, D, n, kind):
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, kind, n, padding=0.1), gradients(n, D, torch.float16, 8, extra=4)
    scale = float(np.float32(0.7))
    names, sums, mags = reference(keys, d, scale, PAD)
    dense, dense_mags = torch.zeros(R, D, dtype=torch.float64, device=DEV), torch.zeros(R, D, dtype=torch.float64, device=DEV)
    dense[names], dense_mags[names] = sums, mags
    dE = torch.full((R, D), float("nan"), device=DEV)
    tab.ctx.embed_grad_dense(keys, d, dE, scale=scale, padding=PAD)
    close(dE, dense, dense_mags, n)
    assert bool((dE[torch.isin(torch.arange(R, device=DEV), names, invert=True)] == 0).all())
    old = torch.randn(R, D, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    dE = old.clone()
    tab.ctx.embed_grad_dense(keys, d, dE, scale=scale, padding=PAD, accumulate=True)
    close(dE, dense + old.double(), dense_mags + old.double().abs(), n)
    away = torch.isin(torch.arange(R, device=DEV), names, invert=True)
    assert torch.equal(dE[away], old[away]) and tab.ctx.status() == 0


@pytest.mark.parametrize("n", [5, 700, 3000, 20000, 70001])
@pytest.mark.parametrize("where", ["first", "last"])
def test_a_bad_token_rejects_the_batch(n, where):
    R, D = 1 << 10, 36
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, "text", n), gradients(n, D, torch.float32, 2)
    bad = keys.clone()
    bad[0 if where == "first" else n - 1] = R if where == "first" else -1
    names, grads = run_grad(tab, bad, d)
    assert len(names) == 0 and tab.ctx.status() == ECRM_EKEYRANGE
    for accumulate in (False, True):
        dE = torch.full((R, D), 3.0, device=DEV)
        tab.ctx.embed_grad_dense(bad, d, dE, accumulate=accumulate)
        assert bool((dE == (3.0 if accumulate else 0.0)).all())
    tab.ctx.clear_status()
    check_grad(tab, keys, d)                              # the next call starts clean
    assert tab.ctx.status() == 0


def test_differences():
    """Small steps of the table in powers of two, so that nothing is rounded: the gradient is what the loss changes by."""
    R, D, n, scale, h = 64, 12, 500, 4.0, 2.0 ** -4
    tab = Table(R, D, max_batch=n)
    rng = np.random.default_rng(5)
    tab.E[:] = torch.from_numpy(rng.integers(-32, 33, (R, D)) / 64.0).to(DEV)
    keys = tokens(R, n, "text", 4, padding=0.1)
    w = torch.from_numpy(rng.integers(-16, 17, (n, D)) / 16.0).to(DEV).float()

    def loss():
        out = torch.empty(n, D, device=DEV)
        tab.ctx.embed(keys, out, scale=scale, padding=PAD)
        return float((out.double() * w.double()).sum())

    dE = torch.empty(R, D, device=DEV)
    tab.ctx.embed_grad_dense(keys, w, dE, scale=scale, padding=PAD)
    for x in [0, 1, 2, 17, R - 1]:
        for c in (0, 5, D - 1):
            at = float(tab.E[x, c])
            tab.E[x, c] = at + h
            up = loss()
            tab.E[x, c] = at - h
            down = loss()
            tab.E[x, c] = at
            assert (up - down) / (2 * h) == float(dE[x, c])


def test_other_calls_in_between_keep_their_results():
    """Updates, statistics and reads around gradient calls that share the scratch buffer with them."""
    R, D, n = 4 * 2000, 64, 40000
    a, b = Table(R, D, max_batch=n, seed=9), Table(R, D, max_batch=n, seed=9)
    for i, m in enumerate((n, 3000, 50)):
        keys, g = tokens(R, m, "text", i), gradients(m, D, torch.float32, i).contiguous()
        for tab in (a, b):
            tab.ctx.update(keys, g)
        stats = b.ctx.batch_stats()
        check_grad(b, keys, gradients(m, D, torch.bfloat16, i))
        assert b.ctx.batch_stats() == stats
        for x, y in ((a.E, b.E), (a.A, b.A), (a.PE, b.PE), (a.PA, b.PA), (a.load, b.load)):
            assert torch.equal(x, y)


class Large:
    """A table of zeros, too large to be filled for a test."""

    def __init__(self, R, D, max_batch):
        self.R, self.D = R, D
        self.E, A = torch.zeros(R, D, device=DEV), torch.empty(R, D, device=DEV)
        P, load = torch.empty(2, R // 4, D, device=DEV), torch.zeros(2, 5, dtype=torch.int64, device=DEV)
        self.ctx = Ecrm(R, D, max_batch=max_batch)
        scratch = torch.empty(self.ctx.scratch_bytes(), dtype=torch.uint8, device=DEV)
        self.ctx.bind(self.E, A, P[0], P[1], load[0], load[1], scratch)


def test_rows_beyond_32_bit_offsets():
    R, D, n = 1 << 28, 16, 5000                           # 2^32 floats to a table
    tab = Large(R, D, n)
    rng = np.random.default_rng(1)
    rows = np.unique(np.concatenate([[0, 1, R - 1, R - 2, 1 << 27, (1 << 27) - 1], rng.integers(0, R, 500)]))
    at = torch.from_numpy(rows).to(DEV)
    tab.E[at] = torch.randn(len(rows), D, device=DEV)
    keys = at[torch.from_numpy(rng.integers(0, len(rows), n)).to(DEV)]
    out = torch.empty(n, D, device=DEV)
    tab.ctx.embed(keys, out)
    assert torch.equal(out, tab.E[keys])
    d = gradients(n, D, torch.float32, 1)
    names, sums, mags = check_grad(tab, keys, d)
    tab.E.zero_()
    tab.ctx.embed_grad_dense(keys, d, tab.E, accumulate=True)
    close(tab.E[names], sums, mags, n)
    assert int((tab.E[:, 0] != 0).sum()) <= len(names)
    tab.ctx.embed_grad_dense(keys, d, tab.E)
    close(tab.E[names], sums, mags, n)
    assert tab.ctx.status() == 0


def test_tokens_beyond_32_bit_offsets():
    """Gradients of looked-up rows, and looked-up rows, that lie more than 2^32 bytes and 2^31 elements into their memory."""
    R, D, n = 1 << 12, 1024, (1 << 21) + 77
    tab = Large(R, D, n)
    tab.E[:] = torch.randn(R, D, device=DEV)
    keys = torch.full((n,), PAD, dtype=torch.int64, device=DEV)
    keys[-500:] = torch.randint(0, R, (500,), device=DEV)
    keys[:3] = 5
    d = torch.empty(n, D, dtype=torch.bfloat16, device=DEV)
    d[:3], d[-500:] = torch.randn(3, D, device=DEV), torch.randn(500, D, device=DEV)
    ok, og = torch.empty(n, dtype=torch.int64, device=DEV), torch.empty(n, D, device=DEV)
    count = torch.zeros(1, dtype=torch.int64, device=DEV)
    tab.ctx.embed_grad(keys, d, ok, og, count, padding=PAD)
    some = torch.cat([torch.arange(3, device=DEV), torch.arange(n - 500, n, device=DEV)])
    names, sums, mags = reference(keys[some], d[some], 1.0, PAD)
    u = int(count)
    assert torch.equal(ok[:u], names) and bool((ok[u:] == -1).all())
    close(og[:u], sums, mags, n)
    d.fill_(7.0)
    tab.ctx.embed(keys, d, padding=PAD)
    assert torch.equal(d[-500:], tab.E[keys[-500:]].to(torch.bfloat16)) and not bool(d[1000:2000].any())
    assert tab.ctx.status() == 0


def test_during_a_recovery():
    """Gradients between the calls of a recovery, whose updates wait in their buffer meanwhile: the tables end as without them; a
    lookup sees what a degraded read sees."""
    R, D, n, cap = 4 * 1000, 64, 3000, 4000
    a, b = Table(R, D, max_batch=n + cap, seed=9), Table(R, D, max_batch=n + cap, seed=9)
    for tab in (a, b):
        bk, bg = torch.empty(2 * cap, dtype=torch.int64, device=DEV), torch.empty(2 * cap, D, device=DEV)
        tab.ctx.fail_server(2)
        tab.ctx.recovery_begin(2, 2, bk, bg, cap)
        for step in range(2):
            keys, g = tokens(R, n // 2, "uniform", step), gradients(n // 2, D, torch.float32, step).contiguous()
            tab.ctx.recovery_lock()
            tab.ctx.update(keys, g)
            if tab is b:
                waiting = b.ctx.recovery_state()
                check_grad(b, tokens(R, 5000, "text", 7), gradients(5000, D, torch.bfloat16, 7))
                read, out = torch.empty(n // 2, D, device=DEV), torch.empty(n // 2, D, device=DEV)
                b.ctx.degraded_read(keys, 2, read)
                b.ctx.embed(keys, out, lost_server=2)
                assert torch.equal(read, out) and b.ctx.recovery_state() == waiting
            tab.ctx.recovery_decode()
            tab.ctx.recovery_unlock()
        assert tab.ctx.status() == 0 and not tab.ctx.recovery_state()["active"]
    for x, y in ((a.E, b.E), (a.A, b.A), (a.PE, b.PE), (a.PA, b.PA), (a.load, b.load)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("n", [200, 1500, 5000, 40000, 100000])
def test_in_a_graph(n):
    """Replays on new contents, with the program's own calls on the same context in between."""
    R, D = 1 << 12, 128
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, "text", 1, padding=0.1), gradients(n, D, torch.bfloat16, 1).contiguous()
    out, ok, og = torch.empty(n, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, dtype=torch.int64, device=DEV), torch.empty(n, D, device=DEV)
    count, dE = torch.empty(1, dtype=torch.int64, device=DEV), torch.empty(R, D, device=DEV)

    def step(stream=None):
        tab.ctx.embed(keys, out, scale=2.0, padding=PAD, stream=stream)
        tab.ctx.embed_grad(keys, d, ok, og, count, scale=2.0, padding=PAD, stream=stream)
        tab.ctx.embed_grad_dense(keys, d, dE, scale=2.0, padding=PAD, stream=stream)

    step()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for rep in range(4):
        keys.copy_(tokens(R, n, ("uniform", "one", "text", "runs")[rep], rep, padding=0.1))
        d.copy_(gradients(n, D, torch.bfloat16, 20 + rep))
        ok.fill_(5), og.fill_(5.0), out.fill_(5.0), dE.fill_(5.0)
        graph.replay()
        got = [x.clone() for x in (out, ok, og, count, dE)]
        ok.fill_(5), og.fill_(5.0), out.fill_(5.0), dE.fill_(5.0)
        step()
        for x, y in zip(got, (out, ok, og, count, dE)):
            assert torch.equal(x, y), rep
        torch.cuda.synchronize()
    assert tab.ctx.status() == 0


def test_on_another_stream():
    R, D, n = 1 << 12, 128, 20011
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, "text", 1), gradients(n, D, torch.float16, 1)
    want = run_grad(tab, keys, d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run_grad(tab, keys, d)
        out = torch.empty(n, D, device=DEV)
        tab.ctx.embed(keys, out)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(out, tab.E[keys])


def test_refusals():
    R, D, n = 1 << 10, 36, 100
    tab = Table(R, D, max_batch=n)
    keys = tokens(R, n + 1, "uniform", 1)
    ok, og, count = torch.zeros(n + 1, dtype=torch.int64, device=DEV), torch.zeros(n + 1, D, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    d = torch.zeros(n + 1, 2 * D, dtype=torch.bfloat16, device=DEV)

    def refused(code, call, *a, **kw):
        with pytest.raises(EcrmError) as e:
            call(*a, **kw)
        assert e.value.code == code

    refused(ECRM_EBATCH, tab.ctx.embed_grad, keys, d[:, :D], ok, og, count)
    k = keys[:n]
    refused(ECRM_EINVAL, tab.ctx.embed_grad, k, d[:n, :D], ok, og, count, scale=float("nan"))
    refused(ECRM_EINVAL, tab.ctx.embed_grad, k, d[:n, 2:D + 2], ok, og, count)                      # not aligned to four elements
    refused(ECRM_EINVAL, tab.ctx.embed_grad, k, torch.zeros(n, D + 2, device=DEV)[:, :D], ok, og, count)    # rows that are not
    refused(ECRM_EINVAL, tab.ctx.embed, k, d[:n, 2:D + 2])
    refused(ECRM_EINVAL, tab.ctx.embed, k, d[:n, :D], lost_server=5)
    refused(ECRM_EINVAL, tab.ctx.embed, k, d[:n, :D], scale=float("inf"))
    with pytest.raises(AssertionError):
        tab.ctx.embed(k, d[:n, :D + 4])
    with pytest.raises(KeyError):
        tab.ctx.embed(k, torch.zeros(n, D, dtype=torch.float64, device=DEV))
    assert not og.any() and not ok.any() and tab.ctx.status() == 0
    none = keys[:0]
    count.fill_(9)
    tab.ctx.embed_grad(none, d[:0, :D], ok, og, count)
    tab.ctx.embed(none, d[:0, :D])
    dE = torch.ones(R, D, device=DEV)
    tab.ctx.embed_grad_dense(none, d[:0, :D], dE, accumulate=True)
    assert int(count) == 0 and bool((dE == 1).all())
    tab.ctx.embed_grad_dense(none, d[:0, :D], dE)
    assert bool((dE == 0).all()) and tab.ctx.status() == 0


def fresh(R=1 << 10, D=36, n=64):
    """A context that has been bound and encoded, whose next call is its first one; the scratch buffer held anything."""
    tab = Table(R, D, max_batch=n)
    bad = torch.full((n,), R, dtype=torch.int64, device=DEV)
    torch.cuda.synchronize()
    return tab, bad, torch.zeros(n, D, device=DEV)


def test_a_first_lookup_on_another_stream_clears_nothing():
    """The lookup is held up on its stream until an update behind it on the main one has found a bad key."""
    tab, bad, grads = fresh()
    keys, out = tokens(tab.R, 64, "uniform", 1), torch.empty(64, tab.D, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        tab.ctx.embed(keys, out)
    tab.ctx.update(bad, grads)
    torch.cuda.current_stream().synchronize()
    side.synchronize()
    assert tab.ctx.status() == ECRM_EKEYRANGE and tab.ctx.batch_stats()["rejected"] == 1
    assert torch.equal(out, tab.E[keys])


def test_a_first_lookup_in_a_graph_clears_nothing_when_it_is_replayed():
    tab, bad, grads = fresh()
    keys, out = tokens(tab.R, 64, "uniform", 1), torch.empty(64, tab.D, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tab.ctx.embed(keys, out)
    tab.ctx.update(bad, grads)
    for _ in range(3):
        out.fill_(5.0)
        graph.replay()
        assert tab.ctx.status() == ECRM_EKEYRANGE and tab.ctx.batch_stats()["rejected"] == 1
        assert torch.equal(out, tab.E[keys])
    tab.ctx.clear_status()
    graph.replay()
    assert tab.ctx.status() == 0


@pytest.mark.parametrize("D", [8, 36, 128])
def test_distinct_keys_in_the_tokens_place(D):
    """... or over a part of them: the tokens have been read by then, in batches of every size."""
    tab = Table(1 << 11, D, max_batch=70001)
    for n in (1, 2, 64, 200, 256, 257, 2000, 9000, 70001):
        keys, d = tokens(tab.R, n, "text", n, padding=0.1), gradients(n, D, torch.bfloat16, 1)
        names, grads = run_grad(tab, keys, d)
        for shift in (0, 1):
            words = torch.full((n + 1,), 77, dtype=torch.int64, device=DEV)
            words[:n] = keys
            og, count = torch.full((n, D), 77.0, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
            tab.ctx.embed_grad(words[:n], d, words[shift:shift + n], og, count, padding=PAD)
            u = int(count)
            assert torch.equal(words[shift:shift + u], names) and bool((words[shift + u:shift + n] == -1).all())
            assert torch.equal(og[:u], grads) and bool((og[u:] == 77.0).all())
    assert tab.ctx.status() == 0


def test_overlaps_are_refused():
    D, n = 36, 100
    tab = Table(1 << 10, D, max_batch=n)
    bytes_ = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)

    def at(byte, shape, dtype):
        size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        return bytes_[byte:byte + size].view(dtype).view(shape)

    row = 4 * D
    keys, wide = at(0, (n,), torch.int64), at(1024, (n, 4 * D), torch.float32)
    d, behind = wide[:, D:2 * D], 1024 + n * 4 * row
    ok, og, count = at(behind, (n,), torch.int64), at(behind + 1024, (n, D), torch.float32), at(behind + 1024 + n * row, (1,), torch.int64)
    tab.ctx.embed_grad(keys, d, ok, og, count)           # one behind the other
    assert int(count) == 1 and tab.ctx.status() == 0
    bytes_.zero_()
    word = lambda byte: at(byte, (1,), torch.int64)  # noqa: E731
    words, rows = (lambda byte: at(byte, (n,), torch.int64)), (lambda byte: at(byte, (n, D), torch.float32))
    last = 1024 + (n - 1) * 4 * row + 2 * row            # behind the last row of d
    bad = [(ok, rows(n * 8 - 16), count), (ok, rows(1024), count), (ok, rows(1024 + row - 16), count), (ok, rows(last - 16), count),
           (words(1024 + row), og, count), (words(last - 8), og, count), (words(behind + 1024 - 792), og, count), (words(behind + 1024 + n * row - 8), og, count),
           (ok, og, word(0)), (ok, og, word(n * 8 - 8)), (ok, og, word(1024 + row)), (ok, og, word(last - 8)), (ok, og, word(behind)),
           (ok, og, word(behind + 1024 + 8))]
    for a, b, c in bad:
        assert tab.ctx.embed_grad(keys, d, a, b, c, check=False) == ECRM_EINVAL
    assert tab.ctx.embed_grad(keys, d, ok, og, word(last)) == 0 and tab.ctx.embed_grad(keys, d, ok, og, word(n * 8)) == 0
    assert tab.ctx.embed_grad(keys, d, ok, og, word(1024 + 3 * 4 * row + 2 * row)) == 0       # between two rows of d
    bytes_.zero_()
    for byte in (0, n * 8 - 8):
        assert tab.ctx.embed(at(byte, (n,), torch.int64), at(0 if byte else 512, (n, D), torch.float32), check=False) == ECRM_EINVAL
    dE = at(1 << 18, (1 << 10, D), torch.float32)
    for accumulate in (False, True):
        assert tab.ctx.embed_grad_dense(at(1 << 18, (n,), torch.int64), d, dE, accumulate=accumulate, check=False) == ECRM_EINVAL
        assert tab.ctx.embed_grad_dense(keys, dE[:n], dE, accumulate=accumulate, check=False) == ECRM_EINVAL
        assert tab.ctx.embed_grad_dense(keys, d, dE, accumulate=accumulate) == 0
    assert tab.ctx.status() == 0 and not bytes_.any()


def test_a_context_without_room_for_gradients():
    """... updates and looks up in the smaller scratch buffer as any other, and refuses the gradient calls."""
    R, D, n = 4 * 500, 1024, 3000
    a, b = Table(R, D, max_batch=n, seed=9), Table(R, D, max_batch=n, seed=9)
    size = b.ctx.update_scratch_bytes()
    assert size < b.ctx.scratch_bytes()
    args = (b.E, b.A, b.PE, b.PA, b.load[0], b.load[1])
    with pytest.raises(EcrmError) as e:
        b.ctx.bind(*args, b.scratch[:size - 1])
    assert e.value.code == ECRM_ESCRATCH
    b.scratch.fill_(0xA5)
    b.ctx.bind(*args, b.scratch[:size])
    keys, g = tokens(R, n, "text", 1), gradients(n, D, torch.float32, 2).contiguous()
    ok, og, count = torch.full((n,), 7, dtype=torch.int64, device=DEV), torch.full((n, D), 7.0, device=DEV), torch.full((1,), 7, dtype=torch.int64, device=DEV)
    dE = torch.full((R, D), 7.0, device=DEV)
    for m in (n, 1):
        for tab in (a, b):
            tab.ctx.update(keys[:m], g[:m])
        assert b.ctx.embed_grad(keys[:m], g[:m], ok, og, count, check=False) == ECRM_ESCRATCH
        assert b.ctx.embed_grad_dense(keys[:m], g[:m], dE, check=False) == ECRM_ESCRATCH
    for x in (ok, og, count, dE):
        assert bool((x == 7).all())
    for x, y in ((a.E, b.E), (a.A, b.A), (a.PE, b.PE), (a.PA, b.PA), (a.load, b.load)):
        assert torch.equal(x, y)
    out = torch.empty(n, D, device=DEV)
    b.ctx.embed(keys, out)
    assert torch.equal(out, b.E[keys]) and a.ctx.status() == b.ctx.status() == 0
    assert bool((b.scratch[size:] == 0xA5).all())
    b.ctx.bind(*args, b.scratch[:b.ctx.scratch_bytes()])
    check_grad(b, keys, g)


@pytest.mark.parametrize("R,D,n,kind", [(1 << 20, 128, (1 << 21) + (1 << 18), "uniform"), (1 << 18, 128, (1 << 21) + 100003, "text"),
                                        (1 << 20, 256, 2100003, "uniform")])
def test_counts_that_are_added_up_by_a_launch(R, D, n, kind):
    """More than 1024 (2048) groups of workgroups, with rows that begin in all of them."""
    tab = Table(R, D, max_batch=n)
    check_grad(tab, tokens(R, n, kind, n, padding=0.03), gradients(n, D, torch.bfloat16, 5))
    assert tab.ctx.status() == 0


@pytest.mark.parametrize("n", [300007, 2100003])
def test_large_batches_of_padding_and_of_bad_tokens(n):
    """The radix sort whose counts are added up in groups, with four items to a thread and with eight."""
    R, D = 1 << 12, 12
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, "text", n, padding=0.1), gradients(n, D, torch.float32, 2)
    pads, nans = torch.full((n,), PAD, dtype=torch.int64, device=DEV), torch.full((n, D), float("nan"), device=DEV)
    names, grads = run_grad(tab, pads, nans)
    assert len(names) == 0 and tab.ctx.status() == 0
    for accumulate in (True, False):
        dE = torch.full((R, D), 3.0, device=DEV)
        tab.ctx.embed_grad_dense(pads, nans, dE, padding=PAD, accumulate=accumulate)
        assert bool((dE == (3.0 if accumulate else 0.0)).all())
    for where, what in ((0, R), (n // 2, 1 << 40), (n - 1, -1)):
        bad = keys.clone()
        bad[where] = what
        names, grads = run_grad(tab, bad, d)
        assert len(names) == 0 and tab.ctx.status() == ECRM_EKEYRANGE
        for accumulate in (False, True):
            dE = torch.full((R, D), 3.0, device=DEV)
            tab.ctx.embed_grad_dense(bad, d, dE, padding=PAD, accumulate=accumulate)
            assert bool((dE == (3.0 if accumulate else 0.0)).all())
        tab.ctx.clear_status()
        pads[where] = keys[where] = 5                     # one token alone
        names, grads = run_grad(tab, pads, d)
        assert names.tolist() == [5] and torch.equal(grads[0], d[(pads == 5)].double().sum(0).float()) and tab.ctx.status() == 0
        pads[where] = PAD
        check_grad(tab, keys, d)


@pytest.mark.parametrize("n", [300007, 2100003])
def test_large_batches_in_a_graph(n):
    R, D = 1 << 18, 8
    tab = Table(R, D, max_batch=n)
    keys, d = tokens(R, n, "text", 1, padding=0.1), gradients(n, D, torch.bfloat16, 1)
    ok, og = torch.empty(n, dtype=torch.int64, device=DEV), torch.empty(n, D, device=DEV)
    count, dE = torch.empty(1, dtype=torch.int64, device=DEV), torch.empty(R, D, device=DEV)

    def step():
        tab.ctx.embed_grad(keys, d, ok, og, count, padding=PAD)
        tab.ctx.embed_grad_dense(keys, d, dE, padding=PAD)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        keys.copy_(tokens(R, n, ("uniform", "one", "text", "runs")[rep], rep, padding=0.1))
        d.copy_(gradients(n, D, torch.bfloat16, 20 + rep))
        ok.fill_(5), og.fill_(5.0), dE.fill_(5.0)
        graph.replay()
        got = [x.clone() for x in (ok, og, count, dE)]
        ok.fill_(5), og.fill_(5.0), dE.fill_(5.0)
        step()
        for x, y in zip(got, (ok, og, count, dE)):
            assert torch.equal(x, y), rep
        torch.cuda.synchronize()
    assert tab.ctx.status() == 0


def test_strides_beyond_any_memory():
    """... do not matter to a single row, and are refused for more."""
    D = 36
    tab = Table(1 << 10, D, max_batch=4)
    keys, d = torch.tensor([7, 9], device=DEV), torch.ones(2, D, device=DEV)
    out, ok, og, count = torch.zeros(2, D, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV), torch.zeros(2, D, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    dE, lib, raw = torch.zeros(1 << 10, D, device=DEV), tab.ctx._lib, tab.ctx._ctx
    k, none = keys.data_ptr(), 1 << 63
    for n, code in ((2, ECRM_EINVAL), (1, 0)):
        for stride in ((1 << 62), (1 << 64) - 4, (1 << 48) + 4):
            assert lib.ecrm_embed(raw, k, n, none, 1.0, 0xFFFFFFFF, out.data_ptr(), 0, stride, None) == code
            assert lib.ecrm_embed_grad(raw, k, d.data_ptr(), 0, stride, n, none, 1.0, ok.data_ptr(), og.data_ptr(), count.data_ptr(), None) == code
            assert lib.ecrm_embed_grad_dense(raw, k, d.data_ptr(), 0, stride, n, none, 1.0, dE.data_ptr(), 0, None) == code
        assert code == 0 or not (out.any() or og.any() or dE.any())
    assert torch.equal(out[0], tab.E[7]) and int(count) == 1 and int(ok[0]) == 7 and bool((og[0] == 1).all()) and float(dE.sum()) == D
    assert tab.ctx.status() == 0
