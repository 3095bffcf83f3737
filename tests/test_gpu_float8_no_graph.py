"""norm and join to 8 bits and the product of the result, of tensors that require
gradients: the values are those without, and a backward pass through them raises (GPU)."""
import pytest
import torch

import paper_2608_16308_amd as dbs
from paper_2608_16308_amd import Norm

pytestmark = pytest.mark.gpu


def chain(ctx, x, r, w, weight):
    nm, w8 = Norm(weight), ctx.pack8(w, block="tile")
    h8 = ctx.norm(x, nm, to8=True)
    s, k8 = ctx.join(x, r, before=nm, to8=True)
    p8 = ctx.pack8(x)
    return [s, ctx.linear8(h8, w8), ctx.linear8(k8, w8, residual=r[:, :w.shape[0]]), ctx.linear8(p8, w8), ctx.unpack8(k8)]


@pytest.mark.parametrize("t", [3, 70])
def test_chain(t):
    g = torch.Generator(device="cuda")
    g.manual_seed(t)
    made = [torch.randn(s, generator=g, device="cuda").half() for s in ((t, 700), (t, 700), (96, 700), (700,))]
    want = chain(dbs.LayerContext(), *made)
    side = torch.cuda.Stream()
    own = dbs.LayerContext(side)
    for ctx in (dbs.LayerContext(), own):  # (a marked matrix on another stream than its own too)
        leaves = [v.clone().requires_grad_() for v in made]
        side.wait_stream(torch.cuda.current_stream())
        got = chain(ctx, *leaves)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert a.requires_grad and not b.requires_grad and torch.equal(a, b)
            with pytest.raises(dbs.DbsError) as e:
                a.float().sum().backward()
            assert "builds no autograd graph" in str(e.value)
