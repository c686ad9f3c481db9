"""The activations of 32-bit blocks and their derivatives by themselves: with weights of zeros and ones no sum adds an error, so that what a block
returns is the function's own value.

Bounds, in roundings of 32 bits (2^-24 relative): e^x is off by at most 3 steps (6 roundings), erfc by 16 steps (32), a quotient, a product and
a sum by one; an argument's error counts times the function's condition.  For values behind fp32's normal range 2^-120.  The last test shows that
what 16-bit blocks compute would not pass."""
import pytest
import torch

import test_gpu_feed_forward as ff
from paper_2104_01981_amd import FeedForward

R = 2.0 ** -24
SECOND = 1 + 2.0 ** -16                                  # products of errors
KINDS = ["silu", "gelu", "relu"]


def points(rows):
    """Arguments for `rows` rows of three: evenly over what matters, close to zero on either side, around the derivatives' zeros, far
    out."""
    near = torch.cat([s * torch.logspace(-30, 1, max(1, 3 * rows // 8), dtype=torch.float64) for s in (1, -1)])
    zeros = torch.cat([c + torch.linspace(-1e-3, 1e-3, max(1, rows // 8), dtype=torch.float64) for c in (-1.2784645, -0.7517916)])
    far = torch.tensor([0.0, -0.0, 200.0, -200.0, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38], dtype=torch.float64)
    some = torch.cat([far, zeros, near])
    return torch.cat([some, torch.linspace(-110, 110, 3 * rows - len(some), dtype=torch.float64)]).float().view(-1, 3)


def condition(g):
    """How often the argument's relative error counts in that of erfc(-g / sqrt 2)."""
    z = -g * 0.5 ** 0.5
    return z.abs() * 2 / torch.pi ** 0.5 / torch.special.erfcx(z)


def value_bound(kind, g):
    """Of what act(g) is off by; g in 64 bits."""
    if kind == "relu":
        return torch.zeros_like(g)
    share = 6 * torch.sigmoid(-g) + 3 if kind == "silu" else 1.3 * condition(g) + 33
    return share * R * SECOND * ff.value(kind, g).abs() + 2.0 ** -120


def slope_bound(kind, g):
    if kind == "relu":
        return torch.zeros_like(g)
    if kind == "silu":                                   # q (1 + g (1 - q))
        q, p = torch.sigmoid(g), torch.sigmoid(-g)
        of_q = 6 * p + 2
        inner = g.abs() * (of_q * q + 2 * p) + (1 + g * p).abs()
        return (q * inner + (of_q + 1) * q * (1 + g * p).abs()) * R * SECOND + 2.0 ** -120
    q = 0.5 * torch.special.erfc(-g * 0.5 ** 0.5)        # q + g phi(g), phi from e^(-g^2 / 2)
    term = g.abs() * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    off = q * (1.3 * condition(g) + 32) + torch.where(term > 0, term * (g * g / 2 + 9), term) + ff.slope("gelu", g).abs()
    return off * R * SECOND + 2.0 ** -120


def within(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()}, the worst by {float(((got.double() - want).abs() / bound)[bad].max())}"


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [16, 700, 6000])
def test_values_forward(rows, kind):
    """x = (g0, g1, g2, 1), gate weights that take each g, up weights that take the one, down weights that take each h."""
    g = points(rows).to(ff.DEV)
    x = torch.cat([g, torch.ones_like(g[:, :1])], 1)
    wg = torch.eye(4, device=ff.DEV)
    wg[3, 3] = 0.0
    wu = torch.zeros(4, 4, device=ff.DEV)
    wu[:, 3] = 1.0
    out = torch.full_like(x, -7.0)
    FeedForward(wg, wu, torch.eye(4, device=ff.DEV), max_rows=rows, activation=kind).forward(x, out)
    within(out[:, :3], ff.value(kind, g.double()), value_bound(kind, g.double()))
    assert not bool(out[:, 3].any())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [16, 700, 6000])
def test_values_and_derivatives_backward(rows, kind):
    """b = 1 and u = 1, so that dg is the derivative and du the value; d_x is one of them at a time."""
    g = points(rows).to(ff.DEV)
    g = torch.cat([g, g.flip(0)[:, :1]], 1)
    x, d, saved = torch.ones_like(g), torch.ones_like(g), torch.cat([g, torch.ones_like(g)], 1)
    one, none = torch.eye(4, device=ff.DEV), torch.zeros(4, 4, device=ff.DEV)
    d_x = torch.full_like(x, -7.0)
    FeedForward(one, none, one, max_rows=rows, activation=kind, training=True).backward(x, saved, d, d_x)
    within(d_x, ff.slope(kind, g.double()), slope_bound(kind, g.double()))
    FeedForward(none, one, one, max_rows=rows, activation=kind, training=True).backward(x, saved, d, d_x)
    within(d_x, ff.value(kind, g.double()), value_bound(kind, g.double()))


def test_the_bounds_tell_16_bit_forms_from_those():
    """A logistic function from 2^x of a rounded argument and an erf that is good to 1.5e-7 miss the bounds, those of libm do not."""
    g = points(6000)
    g = g[g.abs() <= 80]
    quick = g / (1 + torch.exp2(g * -1.44269504))
    x = g.abs() * 0.70710678
    t = 1 / (1 + 0.3275911 * x)
    tail = 0.5 * t * (0.254829592 + t * (-0.284496736 + t * (1.421413741 + t * (-1.453152027 + t * 1.061405429)))) * torch.exp2(x * x * -1.44269504)
    short = g * torch.where(g < 0, tail, 1 - tail)
    for kind, form in (("silu", quick), ("gelu", short)):
        with pytest.raises(AssertionError):
            within(form, ff.value(kind, g.double()), value_bound(kind, g.double()))
    within(g / (1 + torch.exp(-g)), ff.value("silu", g.double()), value_bound("silu", g.double()))
    within(0.5 * g * torch.special.erfc(g * -0.70710678), ff.value("gelu", g.double()), value_bound("gelu", g.double()))
    q = 1 / (1 + torch.exp(-g))
    within(q * (1 + g * (1 - q)), ff.slope("silu", g.double()), slope_bound("silu", g.double()))
    q = 0.5 * torch.special.erfc(g * -0.70710678)
    within(q + g * torch.exp(-0.5 * g * g) * 0.39894228, ff.slope("gelu", g.double()), slope_bound("gelu", g.double()))
