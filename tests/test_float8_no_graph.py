"""A result that autograd follows back to a call with 8-bit results raises (CPU only:
the library's functions are stood in for and compute nothing)."""
import pytest
import torch

from paper_2608_16308_amd import DbsError, Norm, edges, float8
from paper_2608_16308_amd._lib import DBS_ERR_UNSUPPORTED

BF = torch.bfloat16


class Nothing:
    def __getattr__(self, name):
        return lambda *args: 0


class Context(edges.EdgeOps, float8.Float8Ops):
    def __init__(self):
        self._torch, self.device, self._h, self._fn = torch, torch.device("cpu"), None, Nothing()

    def _call(self, body, inputs):
        return body()


def z(*shape, grad=False):
    return torch.zeros(shape, dtype=BF).requires_grad_(grad)


def raises(out, word):
    assert out.requires_grad
    with pytest.raises(DbsError) as e:
        out.float().sum().backward()
    assert e.value.status == DBS_ERR_UNSUPPORTED and word in str(e.value)


def results(c):
    """8-bit matrices [6, 256] of a leaf that requires a gradient."""
    x, r = z(6, 256, grad=True), z(6, 256)
    yield c.norm(x, Norm(), to8=True)
    yield c.norm(x[2:].expand(4, 256), Norm(), to8=True)
    yield c.norm(r, Norm(z(256, grad=True)), to8=True)
    yield c.norm(r, Norm(None, z(256, grad=True)), to8=True)
    yield c.join(x, r, before=Norm(), to8=True)[1]
    yield c.join(r, x, before=Norm(), to8=True)[1]
    yield c.join(r, r.clone(), before=Norm(), gate=z(256, grad=True), to8=True)[1]
    yield c.pack8(x)
    yield c.pack8(z(256, 6, grad=True), across=True)


def test_products_of_what_was_packed():
    c = Context()
    w = c.pack8(z(64, 256), block="tile")
    assert not w.requires_grad and not c.linear8(z(6, 256), w).requires_grad and not c.unpack8(w).requires_grad
    for x8 in results(c):
        assert x8.requires_grad and x8.shape[1] == 256 and x8.codes.dtype == torch.float8_e4m3fn
        raises(c.linear8(x8, w), "linear8_backward")
        raises(c.linear8(x8, w, bias=z(64), residual=z(x8.shape[0], 64, grad=True)), "linear8_backward")
        raises(c.unpack8(x8), "builds no autograd graph")
        # the gradients' own calls take it
        assert not any(v.requires_grad for v in c.linear8_backward(z(x8.shape[0], 64), x8, w, bias=True))
    w8 = c.pack8(z(64, 256, grad=True), block="tile")
    raises(c.linear8(z(6, 256), w8), "linear8_backward")
    raises(c.linear8(c.pack8(z(6, 256)), w8), "linear8_backward")


def test_the_stream_of_a_join_to_8_bits():
    c = Context()
    raises(c.join(z(6, 256, grad=True), z(6, 256), before=Norm(), to8=True)[0], "join_backward")


def test_without_autograd():
    c = Context()
    with torch.no_grad():
        w8, x8 = c.pack8(z(64, 256, grad=True), block="tile"), c.norm(z(6, 256, grad=True), Norm(), to8=True)
        assert not w8.requires_grad and not x8.requires_grad
    assert not c.linear8(x8, w8).requires_grad
    # a result that keeps its mark is used without autograd
    x8 = c.pack8(z(6, 256, grad=True))
    with torch.no_grad():
        assert not c.linear8(x8, w8).requires_grad
