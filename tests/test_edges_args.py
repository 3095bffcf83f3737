"""What the norms, joins, dropout and 8-bit products refuse, sizes at their limits
included (CPU only): the binding's checks with CPU and meta tensors, and the C
ABI's over a stand-in for the HIP runtime."""
import pytest
import torch

import fake_hip
from paper_2608_16308_amd import Blocks8, DbsError, Norm, edges, float8
from paper_2608_16308_amd._lib import DBS_ERR_ARG, DBS_ERR_UNSUPPORTED

CPU = torch.device("cpu")
META = torch.device("meta")
BF = torch.bfloat16


def rejects(fn, *args, status=DBS_ERR_ARG, **kw):
    with pytest.raises(DbsError) as e:
        fn(*args, **kw)
    assert e.value.status == status
    return str(e.value)


class Context(edges.EdgeOps, float8.Float8Ops):
    """The binding without a device: a call that comes through its checks says so."""

    def __init__(self, device=CPU):
        self._torch, self.device = torch, device

    def _call(self, body, inputs):
        raise NotImplementedError


def passes(fn, *args, **kw):
    with pytest.raises(NotImplementedError):
        fn(*args, **kw)


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def test_norm():
    c = Context()
    x, nm = z(6, 16), Norm(z(16), z(16), kind="layer", eps=0.0)
    passes(c.norm, x, nm)
    passes(c.norm, x[:, 3:9], Norm())
    passes(c.norm, x[0], nm)
    passes(c.norm, x, nm, y=x)
    passes(c.norm, x, nm, to8=True)
    rejects(c.norm, None, nm)
    rejects(c.norm, x.float(), nm)
    rejects(c.norm, x.t(), nm)
    rejects(c.norm, x, None)
    rejects(c.norm, x, z(16))
    rejects(c.norm, x, Norm(z(15)))
    rejects(c.norm, x, Norm(z(16).half()))
    rejects(c.norm, x, Norm(None, z(32)[::2]))
    rejects(c.norm, x, Norm(kind="batch"))
    for eps in (-1e-6, float("inf"), float("nan")):
        rejects(c.norm, x, Norm(eps=eps))
    rejects(c.norm, x, nm, y=z(6, 15))
    rejects(c.norm, x, nm, y=z(6, 16), to8=True)
    buf = z(200)
    rejects(c.norm, buf[:96].view(6, 16), nm, y=buf[8:104].view(6, 16))
    rejects(c.norm, x, Norm(buf[:16]), y=buf[8:104].view(6, 16))
    passes(c.norm_backward, x, x, nm, add=x)
    rejects(c.norm_backward, x, z(6, 15), nm)
    rejects(c.norm_backward, x, x.half(), nm)
    rejects(c.norm_backward, x, x, None)
    rejects(c.norm_backward, x, x, nm, add=z(5, 16))


def test_join():
    c = Context()
    x, r, nm = z(6, 16), z(6, 16), Norm(z(16))
    passes(c.join, x, r)
    passes(c.join, x, r, after=nm, before=nm, gate=z(16), p=0.5, rng=(1, 2), stream=r)
    passes(c.join, x, r, gate=z(6, 16))
    passes(c.join, x[0], r[0], before=nm)
    passes(c.join, x, r, p=0.0)
    for p in (-0.1, 1.1, float("nan")):
        rejects(c.join, x, r, p=p, rng=(1, 2))
    rejects(c.join, x, r, p=0.5)
    for rng in ((-1, 0), (0, 1 << 64), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64),
                torch.zeros(4, dtype=torch.int64)[::2], torch.zeros(2, dtype=torch.int64, device=META)):
        rejects(c.join, x, r, p=0.5, rng=rng)
    passes(c.join, x, r, p=0.5, rng=torch.zeros(2, dtype=torch.int64))
    rejects(c.join, x, None)
    rejects(c.join, x, z(6, 15))
    rejects(c.join, x, r.half())
    rejects(c.join, x, r, gate=z(6))
    rejects(c.join, x, r, gate=z(5, 16))
    rejects(c.join, x, r, gate=z(16)[None].expand(6, 16))
    rejects(c.join, x, r, to8=True)
    rejects(c.join, x, r, stream=x)
    rejects(c.join, x, r, before=nm, stream=z(6, 17))
    passes(c.join_backward, x, x, x, x, after=nm, before=nm, gate=z(16))
    passes(c.join_backward, x, None, None, None)
    passes(c.join_backward, None, x, None, x, before=nm)
    rejects(c.join_backward, None, None, x, x)
    rejects(c.join_backward, x, x, x, x)
    rejects(c.join_backward, x, None, x, x, before=nm)
    rejects(c.join_backward, x, None, None, None, gate=z(16))
    rejects(c.join_backward, x, None, None, None, after=nm)
    rejects(c.join_backward, x, x, x, None, before=nm)
    rejects(c.join_backward, x, z(6, 15), x, x, before=nm)


def test_dropout():
    c = Context()
    x = z(6, 16)
    passes(c.dropout, x, 0.5, (1, 2))
    passes(c.dropout, x, 0.0, None)
    passes(c.dropout, x[1], 1.0, (1, 2), y=x[1])
    rejects(c.dropout, x, 0.5, None)
    rejects(c.dropout, x, 2.0, (1, 2))
    for rng in (5, (5,), (1, 2, 3), (1.5, 2), "ab", (1, -2), (1 << 64, 0), z(2), torch.zeros(3, dtype=torch.int64)):
        rejects(c.dropout, x, 0.5, rng)
    rejects(c.dropout, x.float(), 0.5, (1, 2))
    buf = z(200)
    rejects(c.dropout, buf[:96].view(6, 16), 0.5, (1, 2), y=buf[8:104].view(6, 16))


def blocks(rows, cols, block="tile", codes=None, exps=None, cd=torch.float8_e4m3fn, ed=torch.uint8, dtype=BF, device=CPU):
    a, b = float8.blocks_shapes(rows, cols, block)
    return Blocks8(torch.zeros(codes or a, dtype=torch.uint8, device=device).view(cd), torch.zeros(exps or b, dtype=ed, device=device), block,
                   (rows, cols), dtype)


def test_blocks():
    c = Context()
    assert float8.blocks_shapes(300, 1000, "row") == ((300, 1024), (300, 8))
    assert float8.blocks_shapes(300, 1000, "tile") == ((300, 1024), (3, 8))
    assert float8.blocks_shapes(0, 5, "tile") == ((0, 128), (0, 4))
    passes(c.pack8, z(6, 16), block="tile", across=True)
    rejects(c.pack8, z(6, 16), block="column")
    rejects(c.pack8, z(6, 16).float())
    ok = blocks(300, 1000)
    passes(c.unpack8, ok)
    passes(c.unpack8, blocks(7, 5, "row"))
    rejects(c.unpack8, z(6, 16))
    for bad in (blocks(300, 1000, codes=(300, 1000)), blocks(300, 1000, exps=(300, 8)), blocks(300, 1000, exps=(3, 7)),
                blocks(300, 1000, cd=torch.uint8), blocks(300, 1000, ed=torch.int8), blocks(300, 1000, dtype=torch.float32),
                Blocks8(ok.codes, ok.exponents, "column", ok.shape, BF), Blocks8(ok.codes, ok.exponents, "tile", (300,), BF),
                Blocks8(torch.zeros(300 * 1024 + 1, dtype=torch.uint8)[1:].view(torch.float8_e4m3fn).view(300, 1024), ok.exponents, "tile",
                        (300, 1000), BF)):
        rejects(c.unpack8, bad)
    rejects(c.unpack8, ok, y=z(300, 999))


def test_products():
    c = Context()
    w, x, x8 = blocks(300, 1000), z(6, 1000), blocks(6, 1000, "row")
    passes(c.linear8, x, w, bias=z(300), residual=z(6, 300))
    passes(c.linear8, x8, w)
    passes(c.linear8, x[0], w)
    rejects(c.linear8, x, z(300, 1000))
    rejects(c.linear8, x, blocks(300, 1000, "row"))
    rejects(c.linear8, blocks(6, 1000, "tile"), w)
    rejects(c.linear8, z(6, 999), w)
    rejects(c.linear8, blocks(6, 999, "row"), w)
    rejects(c.linear8, x.float(), w)
    rejects(c.linear8, x, w, bias=z(299))
    rejects(c.linear8, x, w, residual=z(5, 300))
    rejects(c.linear8, x, w, y=z(6, 301))
    passes(c.linear8_backward, z(6, 300), x, w, bias=True)
    passes(c.linear8_backward, z(6, 300), x8, w)
    passes(c.linear8_backward, z(6, 300), None, w, need_dw=False)
    rejects(c.linear8_backward, z(6, 300), None, w)
    rejects(c.linear8_backward, z(6, 299), x, w)
    rejects(c.linear8_backward, z(6, 300), z(5, 1000), w)
    rejects(c.linear8_backward, z(6, 300), blocks(6, 1000, "row", dtype=torch.float16), w)
    rejects(c.linear8_backward, z(6, 300), x, z(300, 1000))


def test_sizes_that_do_not_fit():
    c = Context(META)
    m = lambda *s: torch.empty(s, dtype=BF, device=META)  # noqa: E731
    for shape in (((1 << 32) + 3, 1), (1, (1 << 32) + 3), ((1 << 30) + 1, 1)):
        for fn in (lambda v: c.norm(v, Norm()), lambda v: c.join(v, v), lambda v: c.dropout(v, 0.5, (1, 2)), c.pack8):
            rejects(fn, m(*shape), status=DBS_ERR_UNSUPPORTED)
        rejects(c.unpack8, blocks(*shape, device=META), status=DBS_ERR_UNSUPPORTED)
    rejects(c.linear8, m(1, (1 << 24) + 1), blocks(1, (1 << 24) + 1, device=META), status=DBS_ERR_UNSUPPORTED)
    rejects(c.linear8_backward, m((1 << 24) + 1, 1), None, blocks(1, 1, device=META), need_dw=False, status=DBS_ERR_UNSUPPORTED)
    rejects(c.linear8_backward, m(1, (1 << 24) + 1), None, blocks((1 << 24) + 1, 1, device=META), need_dw=False, status=DBS_ERR_UNSUPPORTED)


ABI = """
from paper_2608_16308_amd import _lib
L = ctypes.c_void_p()
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0
p = 1 << 20
R = ctypes.byref
norm = lambda kind=1, eps=1e-5, w=p, b=None: R(_lib.NormDesc(kind, eps, w, b))
drop = lambda q=0.5, rng=None: R(_lib.DropDesc(q, 1, 2, rng))
b8 = lambda c=p, e=p: R(_lib.Blocks(c, e))
launches = var("fake_launches")
size = ctypes.c_size_t()
def refused(st, code=1):
    assert st == code and lib.dbs_last_error(), st
    assert launches.value == 0, "something was launched"
def taken(st):
    assert st == 0, lib.dbs_last_error()
    assert launches.value > 0
    launches.value = 0
"""


def test_c_abi():
    fake_hip.run(ABI + """
def nrm(dt=3, t=5, n=64, x=p, ldx=64, d=norm(), y=p, ldy=64, y8=None, L=L):
    return lib.dbs_norm(L, dt, t, n, x, ldx, d, y, ldy, y8)
taken(nrm())
taken(nrm(y=None, y8=b8()))
for bad in (dict(L=None), dict(dt=0), dict(t=-1), dict(x=None), dict(x=p + 1), dict(ldx=63), dict(d=None), dict(d=norm(0)), dict(d=norm(3)),
            dict(d=norm(eps=-1)), dict(d=norm(eps=float("nan"))), dict(d=norm(w=p + 1)), dict(y=None), dict(y8=b8()), dict(ldy=2),
            dict(y=None, y8=b8(c=None)), dict(y=None, y8=b8(c=p + 8)), dict(y=None, y8=b8(e=p + 2))):
    refused(nrm(**bad))
refused(nrm(n=(1 << 30) + 1), 4)
def back(t=5, n=64, dy=p, x=p, d=norm(), add=None, dx=p, dw=p, db=p, work=p, room=1 << 30):
    return lib.dbs_norm_backward(L, 1, t, n, dy, n, x, n, d, add, n, dx, n, dw, db, work, room)
taken(back())
for bad in (dict(dy=None), dict(x=None), dict(d=None), dict(work=None), dict(room=10), dict(work=p + 8), dict(dw=p + 1)):
    refused(back(**bad))
def join(t=5, n=64, branch=p, res=p, after=norm(), before=norm(2), gate=p, ldg=0, d=drop(), s=p, h=p, h8=None):
    return lib.dbs_join(L, 3, t, n, branch, n, res, n, after, before, gate, ldg, 1.0, d, s, n, h, n, h8)
taken(join())
taken(join(after=None, before=None, h=None, gate=None, d=None))
taken(join(ldg=64, h=None, h8=b8()))
for bad in (dict(branch=None), dict(res=None), dict(s=None), dict(before=None), dict(h=None), dict(h8=b8()), dict(ldg=3), dict(gate=p + 1),
            dict(d=drop(1.5)), dict(d=drop(float("nan"))), dict(d=drop(rng=p + 4)), dict(after=norm(5))):
    refused(join(**bad))
def jback(t=5, n=64, ds=p, dh=p, branch=p, s=p, after=norm(), before=norm(2), gate=p, ldg=0, d=drop(), dgate=p, aw=p, ab=None, bw=p, bb=None,
          room=1 << 30):
    return lib.dbs_join_backward(L, 3, t, n, ds, n, dh, n, branch, n, s, n, after, before, gate, ldg, 1.0, d, p, n, p, n, dgate, n, aw, ab, bw, bb,
                                 p, room)
taken(jback())
taken(jback(ds=None))
taken(jback(dh=None, before=None, s=None, bw=None))
for bad in (dict(dh=None), dict(s=None), dict(branch=None), dict(before=None), dict(gate=None), dict(after=None), dict(room=0),
            dict(ds=None, dh=None, before=None, bw=None), dict(aw=p + 1)):
    refused(jback(**bad))
def dropped(t=5, n=64, x=p, d=drop(), y=p):
    return lib.dbs_dropout(L, 3, t, n, x, n, d, y, n)
taken(dropped())
for bad in (dict(x=None), dict(y=None), dict(d=None), dict(d=drop(-0.5))):
    refused(dropped(**bad))
""")


def test_c_abi_of_the_products():
    fake_hip.run(ABI + """
def pack(t=5, n=64, x=p, ldx=64, o=b8()):
    return lib.dbs_pack8(L, 3, t, n, x, ldx, 0, 1, o)
taken(pack())
for bad in (dict(x=None), dict(ldx=63), dict(o=None), dict(o=b8(c=None)), dict(o=b8(c=p + 4)), dict(o=b8(e=p + 1))):
    refused(pack(**bad))
taken(lib.dbs_unpack8(L, 3, 5, 64, 1, b8(), p, 64))
refused(lib.dbs_unpack8(L, 3, 5, 64, 1, None, p, 64))
refused(lib.dbs_unpack8(L, 3, 5, 64, 1, b8(), None, 64))
def lin(t=50, n=640, m=64, x=p, x8=None, w=b8(), bias=p, res=p, y=p, work=p, room=1 << 30):
    return lib.dbs_linear8(L, 3, t, n, m, x, n, x8, w, bias, res, m, y, m, work, room)
taken(lin())
taken(lin(x=None, x8=b8(), work=None, room=0))
taken(lin(t=1))
for bad in (dict(x=None), dict(w=None), dict(w=b8(c=p + 1)), dict(y=None), dict(work=None), dict(room=100), dict(work=p + 8), dict(bias=p + 1)):
    refused(lin(**bad))
refused(lin(n=(1 << 24) + 1), 4)
def lback(t=50, n=640, m=64, dy=p, x=p, x8=None, w=b8(), dx=p, dw=p, db=p, room=1 << 40):
    return lib.dbs_linear8_backward(L, 3, t, n, m, dy, m, x, n, x8, w, dx, n, dw, n, db, p, room)
taken(lback())
taken(lback(x=None, x8=b8()))
taken(lback(x=None, dw=None))
taken(lback(w=None, dx=None))
for bad in (dict(dy=None), dict(x=None), dict(w=None), dict(room=1000), dict(db=p + 1)):
    refused(lback(**bad))
refused(lback(t=(1 << 24) + 1), 4)
""")


def test_launches_of_the_largest_sizes():
    """No launch has 2^32 threads or more, which the runtime refuses."""
    fake_hip.run(ABI + """
big = 1 << 30
most = var("fake_most_threads", ctypes.c_ulong)
room = 1 << 60
calls = []
for t, n in ((big, 1), (1, big), (1 << 20, 1 << 16), (3, 1 << 28)):
    calls += [lambda t=t, n=n: lib.dbs_norm(L, 3, t, n, p, n, norm(), p, n, None),
              lambda t=t, n=n: lib.dbs_norm_backward(L, 3, t, n, p, n, p, n, norm(2), None, n, p, n, p, p, p, room),
              lambda t=t, n=n: lib.dbs_join(L, 3, t, n, p, n, p, n, norm(), norm(), p, 0, 1.0, drop(), p, n, p, n, None),
              lambda t=t, n=n: lib.dbs_join_backward(L, 3, t, n, p, n, p, n, p, n, p, n, norm(), norm(), p, 0, 1.0, drop(), p, n, p, n, p, n, p, p,
                                                     p, p, p, room),
              lambda t=t, n=n: lib.dbs_dropout(L, 3, t, n, p, n, drop(), p, n),
              lambda t=t, n=n: lib.dbs_pack8(L, 3, t, n, p, n, 1, 1, b8()), lambda t=t, n=n: lib.dbs_unpack8(L, 3, t, n, 0, b8(), p, n)]
for t, n, m in ((big, 8, 17), (17, 8, big), (1, 8, big), (16, 1 << 24, 1 << 13), (40, 1 << 24, 40)):
    calls.append(lambda t=t, n=n, m=m: lib.dbs_linear8(L, 3, t, n, m, p, n, None, b8(), p, p, m, p, m, p, room))
for t, n, m in ((1 << 24, 8, 17), (17, big, 1 << 12), (1, 8, 1 << 24)):
    calls.append(lambda t=t, n=n, m=m: lib.dbs_linear8_backward(L, 3, t, n, m, p, m, p, n, None, b8(), p, n, p, n, p, p, room))
for i, f in enumerate(calls):
    most.value = 0
    assert f() == 0, (i, lib.dbs_last_error())
    assert 0 < most.value < 1 << 32, (i, most.value)
""")
