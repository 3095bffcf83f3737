"""The activations and their slopes at infinite arguments, and at finite ones
whose squares are infinite in 32 bits."""
import math

import pytest
import torch

import paper_2608_16308_amd as dbs

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("t", [1, 5, 20, 300])
def test_infinite_arguments(kind, t, dt):
    """act(inf) = inf and act(NaN) = NaN; act(-inf) is what its formula gives:
    -inf, 0 of ReLU, and NaN of the others (an infinity times zero)."""
    ctx = dbs.LayerContext()
    w = torch.zeros((24, 16), dtype=dt, device="cuda")
    w[:, 0] = 1
    x = torch.zeros((t, 16), dtype=dt, device="cuda")
    for z in (math.inf, -math.inf, math.nan):
        x[t - 1, 0] = z
        got = ctx.linear(x, w, act=kind)[t - 1].double()
        if z == math.inf or kind == "none":
            want = z
        else:
            want = 0.0 if z == -math.inf and kind == "relu" else math.nan
        assert torch.equal(torch.nan_to_num(got, nan=123.0, posinf=1e300, neginf=-1e300),
                           torch.nan_to_num(torch.full_like(got, want), nan=123.0, posinf=1e300, neginf=-1e300)), (z, got)
    if dt == torch.bfloat16:  # a gate that passes the largest number of 32 bits, beside an up of one
        x[t - 1, 0] = 2.0 ** 100
        w[:, 0] = 2.0 ** 100
        wu = torch.zeros_like(w)
        wu[:, 0] = 2.0 ** -100
        h = ctx.gated(x, w, wu, act=kind)[t - 1]
        assert bool((h == math.inf).all()), h


@pytest.mark.parametrize("kind", ACTS)
def test_squares_past_32_bits(kind):
    """act(z) is z or 0 and act'(z) one or zero there, in both backward passes."""
    ctx = dbs.LayerContext()
    dt = torch.bfloat16
    z = torch.tensor([1e19, -1e19, 2e19, -2e19, 1e20, -1e20, 3e38, -3e38], device="cuda").to(dt)
    n = len(z)
    value = z.double() if kind == "none" else z.double().clamp(min=0)
    slope = torch.ones_like(value) if kind == "none" else (z > 0).double()
    x, w = torch.ones((1, 1), dtype=dt, device="cuda"), torch.ones((n, 1), dtype=dt, device="cuda")
    assert torch.equal(ctx.linear(z[:, None].contiguous(), x, act=kind)[:, 0].double(), value)
    one = torch.ones((1, n), dtype=dt, device="cuda")
    dx, dw, db = ctx.linear_backward(one, x, w, pre=None if kind == "none" else z[None], act=kind, bias=True)
    assert torch.equal(dw[:, 0].double(), slope) and torch.equal(db.double(), slope) and float(dx) == float(slope.sum())
    dx, dg, du = ctx.gated_backward(one, x, w, torch.zeros_like(w), z[None], one, act=kind)
    assert torch.equal(dg[:, 0].double(), slope) and torch.equal(du[:, 0].double(), value)
    assert float(dx) == float(slope.sum())
