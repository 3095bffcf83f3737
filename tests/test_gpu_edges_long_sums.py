"""Sums of very many equal terms, whose roundings all fall the same way, on the GPU: rows
of 2^28 columns, columns of 2^28 rows."""
import pytest
import torch

import paper_2608_16308_amd as dbs
from paper_2608_16308_amd import Norm

pytestmark = pytest.mark.gpu
DT = torch.float16
HALF = 2.0 ** -11  # half a step of fp16, relative


@pytest.fixture
def ctx():
    yield dbs.LayerContext()
    torch.cuda.empty_cache()


def test_rows(ctx):
    """x = c everywhere: rms gives c / sqrt(c^2 + eps), the gradient of a constant g is
    g rstd eps / (c^2 + eps), the difference of numbers a million times larger."""
    n, c, eps = 1 << 28, 1.375, 1e-6
    x = torch.full((1, n), c, dtype=DT, device="cuda")
    nm = Norm(eps=eps)
    y = ctx.norm(x, nm)
    want = c / (c * c + eps) ** 0.5
    # (2^-20: sums of partial sums, root and products in 32 bits)
    assert float((y.double().amax() - want).abs()) <= (HALF + 2.0 ** -20) * want and float((y.double().amin() - want).abs()) <= (HALF + 2.0 ** -20) * want
    dx, _, _ = ctx.norm_backward(x, x, nm)
    rstd = (c * c + eps) ** -0.5
    want = c * rstd * eps / (c * c + eps)
    # (xh, its square's mean and the product of both: each off by at most 2^-21 of g)
    assert float((dx.double() - want).abs().amax()) <= HALF * want + 3 * 2.0 ** -21 * c * rstd + 2.0 ** -25
    s, h = ctx.join(x, x, before=nm, after=nm)
    want = c / (c * c + eps) ** 0.5 + c
    assert float((s.double() - want).abs().amax()) <= (HALF + 2.0 ** -20) * want
    want /= (want * want + eps) ** 0.5
    assert float((h.double() - want).abs().amax()) <= (HALF + 2.0 ** -20) * want


@pytest.mark.parametrize("n", [8, 5])
def test_columns(ctx, n):
    """Sums over the rows: db of a constant dy, dw with xh that is 1 as nearly as eps allows."""
    rows = 1 << 28
    c = 1.99609375
    dy = torch.full((rows, n), c * 2.0 ** -16, dtype=DT, device="cuda")
    assert float(dy[0, 0]) == c * 2.0 ** -16
    x = torch.full((rows, n), 2.0, dtype=DT, device="cuda")
    w = torch.ones(n, dtype=DT, device="cuda")
    nm = Norm(w, w, kind="rms", eps=0.0)
    # (the sums, about 8160, are in the type's range)
    _, dw, db = ctx.norm_backward(dy, x, nm, need_dx=False)
    for v in (dw, db):
        want = rows * c * 2.0 ** -16
        assert float((v.double() - want).abs().amax()) <= (HALF + 2.0 ** -13) * want, v
