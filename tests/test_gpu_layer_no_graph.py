"""The layers build no autograd graph: a result that a gradient was asked of says
so in the backward pass, and is the same otherwise."""
import pytest
import torch

import paper_2608_16308_amd as dbs
from paper_2608_16308_amd import DbsError
from paper_2608_16308_amd._lib import DBS_ERR_UNSUPPORTED

pytestmark = pytest.mark.gpu


def make(*shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(shape))
    return torch.randn(shape, generator=g, device="cuda").half()


def refuses(out, call):
    assert out.requires_grad
    with pytest.raises(DbsError) as e:
        out.float().sum().backward()
    assert e.value.status == DBS_ERR_UNSUPPORTED and call in str(e.value) and "backward" in str(e.value)


def test_forward():
    ctx = dbs.LayerContext()
    x, w, wu, bias, res = make(20, 64), make(40, 64), make(40, 64), make(40), make(20, 40)
    y, (h, gate, up) = ctx.linear(x, w, bias=bias, residual=res), ctx.gated(x, w, wu, save="full")
    for v in (y, h, gate, up):
        assert not v.requires_grad
    for i in range(4):
        args = [x, w, bias, res]
        args[i] = args[i].clone().requires_grad_()
        got = ctx.linear(args[0], args[1], bias=args[2], residual=args[3])
        assert torch.equal(got.detach(), y)
        refuses(got, "linear")
        assert args[i].grad is None
    for i in range(3):
        args = [x, w, wu]
        args[i] = args[i].clone().requires_grad_()
        got = ctx.gated(*args, save="full")
        for a, b in zip(got, (h, gate, up)):
            assert torch.equal(a.detach(), b)
            refuses(a, "gated")
        refuses(ctx.gated(*args), "gated")
        refuses(ctx.gated(*args, save="8bit")[0], "gated")
    p = w.clone().requires_grad_()
    refuses(ctx.linear(x[0], p), "linear")
    refuses(ctx.linear(x, p, save="full")[1], "linear")
    with torch.no_grad():
        got = ctx.linear(x, p, bias=bias, residual=res)
        assert not got.requires_grad and torch.equal(got, y)


def test_into_a_given_output():
    """The caller's tensors stay as they are, through repeated calls."""
    ctx = dbs.LayerContext()
    x, p, y = make(20, 64), make(40, 64).requires_grad_(), make(20, 40)
    start = y.clone()
    for _ in range(2):
        y.copy_(start)
        got = ctx.linear(x, p, residual=y, y=y)
        assert got.data_ptr() == y.data_ptr() and not y.requires_grad
        refuses(got, "linear")
    assert torch.equal(y, ctx.linear(x, p.detach(), residual=start))
    h = make(20, 40)
    got = ctx.gated(x, p, p, h=h)
    assert got.data_ptr() == h.data_ptr() and not h.requires_grad
    refuses(got, "gated")


def test_beside_gradients_by_hand():
    """Parameters as such in a loop that calls the backward passes itself."""
    ctx = dbs.LayerContext()
    x, p = make(20, 64), make(40, 64).requires_grad_()
    y, pre = ctx.linear(x, p, act="silu", save="full")
    dx, dw, _ = ctx.linear_backward(torch.ones_like(y), x, p, pre=pre, act="silu")
    want = ctx.linear_backward(torch.ones_like(y), x, p.detach(), pre=pre.detach(), act="silu")
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and not dw.requires_grad
