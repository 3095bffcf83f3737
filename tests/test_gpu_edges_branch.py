"""A branch that a join's gradients do not need: its values change nothing (GPU)."""
import pytest
import torch

import paper_2608_16308_amd as dbs
from paper_2608_16308_amd import Norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [7, 1000, 4096, 8192, 20000])
def test_nan_in_a_branch_that_is_not_needed(n):
    ctx = dbs.LayerContext()
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    ds, dh, stream = (torch.randn((9, n), generator=g, device="cuda").bfloat16() for _ in range(3))
    nan = torch.full_like(ds, float("nan"))
    for before in (None, Norm(ds[0].clone(), None)):
        args = dict(before=before, p=0.2, rng=(1, 2))
        grad = None if before is None else dh
        a = ctx.join_backward(ds, grad, nan, stream, **args)
        b = ctx.join_backward(ds, grad, None, stream, **args)
        assert all((u is None) == (v is None) and (u is None or torch.equal(u, v)) for u, v in zip(a, b))
        assert bool(a.branch.isfinite().all())
