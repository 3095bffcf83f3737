"""Joins whose outputs take the place of their inputs, as the C ABI allows it (the stream
that of the residual or the branch, h that of the branch), on the GPU."""
import ctypes

import pytest
import torch

import paper_2608_16308_amd as dbs
from paper_2608_16308_amd import Norm, _lib
from test_gpu_edges import gen, make_norm, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("norms", [("rms", "layer"), (None, "rms"), ("layer", None), (None, None)], ids=str)
@pytest.mark.parametrize("size", [(3, 7), (9, 500), (1100, 1501), (600, 4099), (40, 8200), (300, 16001), (5, 20003)], ids=str)
def test_outputs_in_place(size, norms, dt):
    ctx, g, (t, n) = dbs.LayerContext(), gen(size[1]), size
    after, before = (None if k is None else make_norm(g, n, dt, k) for k in norms)
    branch, residual = rnd(g, size, dt), rnd(g, size, dt)
    stream, h = ctx.join(branch, residual, after=after, before=before, p=0.2, rng=(5, 6))
    desc = lambda v: None if v is None else ctypes.byref(_lib.NormDesc({"rms": 1, "layer": 2}[v.kind], v.eps, v.weight.data_ptr(), v.bias.data_ptr()))  # noqa: E731
    drop = _lib.DropDesc(0.2, 5, 6, None)
    lib = dbs.lib()
    for s_of, h_of in (("residual", None), ("branch", None), (None, "branch"), ("residual", "branch")):
        if h_of and before is None:
            continue
        b, r, s, k = branch.clone(), residual.clone(), torch.full_like(branch, 7.0), torch.full_like(branch, 7.0)
        s = {"residual": r, "branch": b}.get(s_of, s)
        k = b if h_of else k
        st = lib.dbs_join(ctx._h, _lib.DBS_BF16 if dt == torch.bfloat16 else _lib.DBS_F16, t, n, b.data_ptr(), n, r.data_ptr(), n, desc(after),
                          desc(before), None, 0, 1.0, ctypes.byref(drop), s.data_ptr(), n, None if before is None else k.data_ptr(), n, None)
        assert st == 0, lib.dbs_last_error()
        assert torch.equal(s, stream), (s_of, h_of)
        assert before is None or torch.equal(k, h), (s_of, h_of)


def test_norm_and_dropout_in_place():
    ctx, g = dbs.LayerContext(), gen(3)
    for n in (7, 1003, 9001, 20003):
        x = rnd(g, (33, n), torch.float16)
        nm = Norm(eps=1e-5, kind="layer")
        a, b = x.clone(), x.clone()
        assert torch.equal(ctx.norm(a, nm, y=a), ctx.norm(x, nm)) and torch.equal(ctx.dropout(b, 0.3, (1, 2), y=b), ctx.dropout(x, 0.3, (1, 2)))
