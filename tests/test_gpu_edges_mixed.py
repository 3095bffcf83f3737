"""Joins whose two norms are of different kinds, and their gradients, on the GPU against
64 bits."""
import pytest
import torch

import edges_ref as ref
import test_gpu_edges as edges
from gpu_helpers import log
from test_gpu_edges import check, check_all, ctx, gen, rnd  # noqa: F401

pytestmark = pytest.mark.gpu
FORMS = [dict(after="rms", before="layer", gate="vector", scale=0.75, p=0.1), dict(after="layer", before="rms", gate="token", scale=1.0, p=0.3),
         dict(after="layer", before="rms", gate=None, scale=-1.5, p=0.0)]
# a wave, teams of waves, two chunks a lane, rows that registers do not hold; ragged ends; rows in turn
SIZES = [(1, 8), (2, 7), (3, 9), (5, 512), (7, 1111), (33, 4096), (2, 5003), (3, 8200), (2, 14336), (2, 20001), (1100, 1501), (525, 5003), (300, 6151)]


@pytest.mark.parametrize("dt", edges.TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_join(ctx, size, dt):  # noqa: F811
    g = gen(size[0] * 11 + size[1])
    log(f"join of mixed norms {size} {dt}")
    for i, form in enumerate(FORMS):
        args = edges.make_join(g, size, dt, form)
        # (the second form far from zero too)
        branch, residual = rnd(g, size, dt, 2.0, (0.5, 60.0, 0.0)[i]), rnd(g, size, dt, 3.0, (0.0, 0.0, 40.0)[i])
        want = ref.join(branch, residual, **args)
        stream, h = ctx.join(branch, residual, **args)
        check(stream, want["stream"], f"{size} {form} stream")
        check(h, want["h"], f"{size} {form} h")
        ds, dh = rnd(g, size, dt), rnd(g, size, dt)
        check_all(ctx.join_backward(ds, dh, branch, stream, **args), ref.join_backward(ds, dh, branch, stream, **args), f"{size} {form}")
