"""The activations and their slopes over the whole range of both types: every
finite number as an argument.

A projection of one term with a weight of one is its argument exactly, so the
bounds are the functions' own, relative to the value, with u = 2^-24:

* a logistic(q) takes q to 6 u of it (a product of up to four roundings), the
  exponential another 2 u |q| from its argument and 2 u of its own; of 1 + e^-q
  the share e^-q / (1 + e^-q) carries that, the sum, the reciprocal and the
  product after it at most 5 u together.  The error of q only counts left of
  zero, where it is |q| (8 u); right of zero |q| e^-q is below 0.37.
* erfc(x) for x = -z / sqrt 2 taken to 2 u changes by (2 x^2 + 1) 2 u left of
  zero and by less than 2 u right of it, where it is above one; the function
  itself is good to 16 units (32 u); two products more.
* e^(-z^2 / 2) is off by 2 u z^2 from its argument and 2 u.

A logistic, erfc or exponential below 2^-125 may be taken as zero on the way."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2608_16308_amd as dbs
from gpu_helpers import log

gpu = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]
u = 2.0 ** -24
LEAST = 2.0 ** -125
C = math.sqrt(8 / math.pi)  # (1 + tanh(q / 2)) / 2 = logistic(q), q = C (z + 0.044715 z^3)


def lost(factor, product):
    """What a factor that is taken as zero costs."""
    return torch.where(factor < LEAST, product.abs(), torch.zeros_like(product))


def logistic(z, kind):
    """(the logistic, its complement, its argument, the argument's slope, the relative error of the logistic)"""
    q, g = (z, torch.ones_like(z)) if kind == "silu" else (C * (z + 0.044715 * z ** 3), C * (1 + 0.134145 * z * z))
    return torch.sigmoid(q), torch.sigmoid(-q), q, g, (8 * (-q).clamp(min=0) + 8) * u


def erfc_rel(z):
    return (2 * z.clamp(max=0) ** 2 + 40) * u


def value(z, kind):
    """(act(z), its bound) for z in 64 bits."""
    if kind == "none":
        return z, torch.zeros_like(z)
    if kind == "relu":
        return z.clamp(min=0), torch.zeros_like(z)
    if kind == "gelu":
        c = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * c, (z * c).abs() * erfc_rel(z) + lost(c, z * c)
    s, _, _, _, rel = logistic(z, kind)
    return z * s, (z * s).abs() * rel + lost(s, z * s)


def slope(z, kind):
    """(act'(z), its bound)."""
    if kind == "none":
        return torch.ones_like(z), torch.zeros_like(z)
    if kind == "relu":
        return (z > 0).double(), torch.zeros_like(z)
    if kind == "gelu":
        c = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        e = torch.exp(-z * z / 2)
        p = z * e / math.sqrt(2 * math.pi)
        return c + p, (c * erfc_rel(z) + p.abs() * (2 * z * z + 8) * u + u * (c + p).abs() + lost(c, c) + lost(e, p))
    s, s1, q, g, rel = logistic(z, kind)
    f = s + z * g * s * s1
    # 1 - s: what s is off by, and a rounding; right of 18 it is zero in 32 bits
    e1 = torch.where(q > 18, s1, s1 * (8 * q.abs() + 8) * u + 5 * u)
    e1 = torch.where(q < 0, s * rel + u, e1)
    return f, s * rel + z.abs() * g * s * (s1 * (rel + 8 * u) + e1) + u * f.abs() + lost(s, s + z.abs() * g * s)


def numbers(dt):
    """Every finite number of a type."""
    v = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(dt)
    return v[v.isfinite()]


@gpu
@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("kind", ACTS)
def test_values(kind, dt):
    ctx = dbs.LayerContext()
    log(f"values {kind} {dt}")
    z = numbers(dt).cuda()
    want, err = value(z.double(), kind)
    one = torch.ones((1, 1), dtype=dt, device="cuda")
    ref.check(ctx.linear(z[:, None].contiguous(), one, act=kind)[:, 0], want, ref.rounded(want, err, dt), f"{kind} {dt}")
    # a column each: the kernels for few tokens (8 terms, one of them not zero)
    w = torch.zeros((len(z), 8), dtype=dt, device="cuda")
    w[:, 0] = z
    for t in (1, 3):
        x = torch.zeros((t, 8), dtype=dt, device="cuda")
        x[:, 0] = 1
        got = ctx.linear(x, w, act=kind)
        ref.check(got[t - 1], want, ref.rounded(want, err, dt), f"{kind} {dt} {t} tokens")
        # gated with a second projection of one
        wu = torch.zeros_like(w)
        wu[:, 0] = 1
        ref.check(ctx.gated(x, w, wu, act=kind)[t - 1], want, ref.rounded(want, err, dt), f"gated {kind} {dt} {t} tokens")


@gpu
@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("kind", ACTS)
def test_slopes(kind, dt):
    ctx = dbs.LayerContext()
    log(f"slopes {kind} {dt}")
    z = numbers(dt).cuda()[None]
    f, ef = value(z[0].double(), kind)
    d, ed = slope(z[0].double(), kind)
    one = torch.ones_like(z)
    w, x = torch.ones((z.shape[1], 1), dtype=dt, device="cuda"), torch.ones((1, 1), dtype=dt, device="cuda")
    # (a factor is rounded, then its gradient, of one term)
    twice = lambda v, e: ref.rounded(v, ref.rounded(v, e, dt), dt)  # noqa: E731
    dw = ctx.linear_backward(one, x, w, pre=None if kind == "none" else z, act=kind)[1]
    ref.check(dw[:, 0], d, twice(d, ed), f"slope {kind} {dt}")
    _, dg, du = ctx.gated_backward(one, x, w, w, z, one, act=kind)
    ref.check(dg[:, 0], d, twice(d, ed), f"gated slope {kind} {dt}")
    ref.check(du[:, 0], f, twice(f, ef), f"gated value {kind} {dt}")


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_the_bounds_see_a_lost_tail(dt):
    """(Values taken as zero left of where 1 + erf or a rounded logistic would
    lose them, and 1 + erf in 32 bits, are outside.)"""
    z = numbers(dt).double()
    for kind, least in (("gelu", -5.1), ("silu", -16.0), ("gelu_tanh", -4.9)):
        want, err = value(z, kind)
        bound = ref.rounded(want, err, dt)
        ref.check(want.to(dt), want, bound, kind)
        with pytest.raises(AssertionError):
            ref.check(torch.where(z < least, torch.zeros_like(z), want).to(dt), want, bound, kind)
    want, err = value(z, "gelu")
    z32 = z.float()
    with pytest.raises(AssertionError):
        ref.check((0.5 * z32 * (1 + torch.erf(z32 * 0.70710678))).to(dt), want, ref.rounded(want, err, dt), "1 + erf")
    for kind in ("silu", "gelu", "gelu_tanh"):
        d, ed = slope(z, kind)
        bound = ref.rounded(d, ed, dt)
        ref.check(d.to(dt), d, bound, kind)
        for wrong in (z > 1e4, z < -4.5):
            with pytest.raises(AssertionError):
                ref.check(torch.where(wrong, torch.zeros_like(z), d).to(dt), d, bound, kind)
