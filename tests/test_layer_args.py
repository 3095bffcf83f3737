"""What the dense layer operators refuse (CPU only): the binding's checks with
CPU tensors, and the C ABI's over a stand-in for the HIP runtime."""
import pytest
import torch

import fake_hip
from paper_2608_16308_amd import Checkpoint, DbsError, layer
from paper_2608_16308_amd._lib import DBS_ERR_ARG

CPU = torch.device("cpu")
BF = torch.bfloat16


def rejects(fn, *args, **kw):
    with pytest.raises(DbsError) as e:
        fn(*args, **kw)
    assert e.value.status == DBS_ERR_ARG
    return str(e.value)


def rows(t, r=None, c=None, dtype=BF):
    return layer.check_rows(t, "t", dtype, CPU, r, c)


def test_rows():
    z = torch.zeros((6, 16), dtype=BF)
    assert rows(z) == 16 and rows(z, 6, 16) == 16 and rows(z[:, 3:9], 6, 6) == 16 and rows(z[::2], 3, 16) == 32
    # a single row or column may have any stride in that direction
    assert rows(z[:1, :5]) == 5 and rows(z[:, :1]) == 16
    assert rows(torch.zeros((0, 4), dtype=BF)) == 4
    rejects(rows, None)
    rejects(rows, z.float())
    rejects(rows, z, 5, 16)
    rejects(rows, z, 6, 15)
    rejects(rows, z[0])
    rejects(rows, z.t())
    rejects(rows, z[:, ::2])
    rejects(rows, z[:1].expand(6, 16))          # rows on top of each other
    rejects(layer.check_rows, z, "t", BF, torch.device("meta"), None, None)


def test_vector_and_names():
    b = torch.zeros(8, dtype=BF)
    layer.check_vector(b, "bias", BF, CPU, 8)
    rejects(layer.check_vector, b, "bias", BF, CPU, 7)
    rejects(layer.check_vector, b.half(), "bias", BF, CPU, 8)
    rejects(layer.check_vector, b[None], "bias", BF, CPU, 8)
    rejects(layer.check_vector, torch.zeros(16, dtype=BF)[::2], "bias", BF, CPU, 8)
    assert layer._choice("silu", layer.ACTS, "act") == 2
    rejects(layer._choice, "swish", layer.ACTS, "act")
    rejects(layer._choice, "fp8", layer.SAVES, "save")
    rejects(layer._dtype_code, torch, torch.zeros(1), "x")
    rejects(layer._dtype_code, torch, None, "x")


def test_checkpoint_parts():
    def ck(codes=(3, 40), exps=(3, 2), cd=torch.int8, ed=torch.uint8, dtype=BF):
        return Checkpoint(torch.zeros(codes, dtype=cd), torch.zeros(exps, dtype=ed), dtype)
    ok = lambda c: layer.check_checkpoint(torch, c, "x", BF, CPU, 3, 40)  # noqa: E731
    ok(ck())
    assert ck().shape == (3, 40) and ck().nbytes() == 126
    for bad in (ck(codes=(3, 41)), ck(codes=(2, 40)), ck(exps=(3, 1)), ck(cd=torch.uint8), ck(ed=torch.int8), ck(dtype=torch.float16),
                Checkpoint(torch.zeros((40, 3), dtype=torch.int8).t(), torch.zeros((3, 2), dtype=torch.uint8), BF)):
        rejects(ok, bad)


def test_output_apart_from_inputs():
    z = torch.zeros(100, dtype=BF)
    a, b = z[:40].view(4, 10), z[40:80].view(4, 10)
    layer._check_apart(a, "y", ((b, "x"), (None, "bias")))
    rejects(layer._check_apart, a, "y", ((z[30:70].view(4, 10), "x"),))
    # columns of one buffer
    w = torch.zeros((6, 40), dtype=BF)
    layer._check_apart(w[:, 10:20], "y", ((w[:, :10], "x"), (w[:, 20:], "residual"), (w[1:5, 30:], "w")))
    for bad in (w[:, :11], w[:, 19:], w[2:4, 12:14], w[:, :]):
        rejects(layer._check_apart, w[:, 10:20], "y", ((bad, "x"),))


def test_c_abi_refusals():
    fake_hip.run("""
from paper_2608_16308_amd import _lib
L = ctypes.c_void_p()
assert lib.dbs_layer_create(None, None) == 1
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0, lib.dbs_last_error()
launches = var("fake_launches")
a = np.zeros(4096, np.uint16)
p = a.ctypes.data
H = lambda *v: ctypes.byref(_lib.Held(*v))
full, held = H(p, 16, None, None), H(None, 0, p, p)
BF, NONE, SILU = 3, 0, 2

def linear(L=L, dt=BF, t=4, n=16, m=8, x=p, ldx=16, w=p, ldw=16, b=p, act=SILU, r=p, ldr=8, y=p, ldy=8, pre=None,
           work=None, size=0):
    return lib.dbs_linear(L, dt, t, n, m, x, ldx, w, ldw, b, act, r, ldr, y, ldy, pre, work, size)
def gated(L=L, dt=BF, t=4, n=16, m=8, x=p, ldx=16, g=p, ldg=16, u=p, ldu=16, act=SILU, h=p, ldh=8, kg=None, ku=None,
          work=None, size=0):
    return lib.dbs_gated(L, dt, t, n, m, x, ldx, g, ldg, u, ldu, act, h, ldh, kg, ku, work, size)
def lback(L=L, dt=BF, t=4, n=16, m=8, dy=p, lddy=8, x=full, w=p, ldw=16, pre=H(p, 8, None, None), act=SILU, dx=p, lddx=16, dw=p,
          lddw=16, db=p, work=4096, size=1 << 20):
    return lib.dbs_linear_backward(L, dt, t, n, m, dy, lddy, x, w, ldw, pre, act, dx, lddx, dw, lddw, db, work, size)
def gback(L=L, dt=BF, t=4, n=16, m=8, dh=p, lddh=8, x=full, g=p, ldg=16, u=p, ldu=16, gate=H(p, 8, None, None),
          up=H(p, 8, None, None), act=SILU, dx=p, lddx=16, dg=p, lddg=16, du=p, lddu=16, work=4096, size=1 << 20):
    return lib.dbs_gated_backward(L, dt, t, n, m, dh, lddh, x, g, ldg, u, ldu, gate, up, act, dx, lddx, dg, lddg, du, lddu,
                                  work, size)
for f in (linear, gated, lback, gback):
    assert f() == 0, (f, lib.dbs_last_error())
none = launches.value
odd = p + 1
bad = [(linear, d) for d in (dict(L=None), dict(dt=0), dict(dt=2), dict(dt=7), dict(t=-1), dict(n=-1), dict(m=-1), dict(x=None),
       dict(x=odd), dict(ldx=15), dict(w=None), dict(ldw=15), dict(b=odd), dict(act=5), dict(act=-1), dict(ldr=7), dict(y=None),
       dict(ldy=7), dict(pre=H(p, 8, p, p)), dict(pre=H(None, 0, p, None)), dict(pre=H(None, 0, None, None)),
       dict(pre=H(p, 7, None, None)), dict(work=4097, size=64))]
bad += [(gated, d) for d in (dict(L=None), dict(dt=1 << 8), dict(g=None), dict(u=None), dict(ldu=3), dict(h=None), dict(ldh=1),
        dict(kg=full), dict(ku=full), dict(kg=H(p, 8, None, None), ku=held), dict(act=9), dict(t=-5))]
bad += [(lback, d) for d in (dict(L=None), dict(dt=0), dict(dy=None), dict(lddy=7), dict(x=None), dict(x=H(p, 15, None, None)),
        dict(x=H(p, 16, p, p)), dict(x=H(None, 0, p, None)), dict(w=None), dict(ldw=1), dict(pre=None),
        dict(pre=H(None, 0, None, None)), dict(act=77), dict(lddx=15), dict(lddw=15), dict(work=None), dict(size=0),
        dict(work=4097), dict(db=odd))]
bad += [(gback, d) for d in (dict(L=None), dict(dt=0), dict(dh=None), dict(x=None), dict(g=None), dict(u=None), dict(gate=None),
        dict(up=None), dict(dg=None), dict(du=None), dict(lddg=15), dict(lddu=15), dict(work=None), dict(size=100), dict(act=-2))]
for f, d in bad:
    assert f(**d) == 1, (f.__name__, d)
    assert lib.dbs_last_error()
assert linear(n=(1 << 30) + 1, ldx=1 << 31, ldw=1 << 31) == 4
size = ctypes.c_size_t()
assert lib.dbs_backward_work(L, 0, SILU, -1, 1, 1, 0, 0, 0, ctypes.byref(size)) == 1
assert lib.dbs_backward_work(L, 0, SILU, 1, 1, 1, 0, 0, 0, None) == 1
assert lib.dbs_forward_work(None, 0, 1, 1, 1, ctypes.byref(size)) == 1
assert lib.dbs_forward_work(L, 0, 1, 1, 1, None) == 1
for name, args in (("dbs_pack", (p, 16, p, p)), ("dbs_unpack", (p, p, p, 16))):
    f = getattr(lib, name)
    assert f(L, BF, 4, 16, *args) == 0
    n = launches.value
    for i in range(len(args)):
        if args[i] == p:
            assert f(L, BF, 4, 16, *args[:i], None, *args[i + 1:]) == 1, (name, i)
    assert f(L, 0, 4, 16, *args) == 1 and f(L, BF, -4, 16, *args) == 1 and f(None, BF, 4, 16, *args) == 1
    assert launches.value == n
# what a call does not use may be missing; empty calls need nothing
assert lback(act=NONE, pre=None) == 0 and lback(dx=None, w=None, ldw=0) == 0 and lback(dw=None, x=None) == 0
assert gback(dx=None, g=None, u=None) == 0 and gback(dg=None, du=None, x=None) == 0
assert linear(t=0, x=None, y=None, r=None) == 0 and linear(m=0, w=None, b=None, r=None, y=None) == 0
assert linear(b=None, r=None, act=NONE) == 0
assert gback(t=0, dh=None, x=None, gate=None, up=None, dx=None) == 0
""")


def test_create_without_memory():
    fake_hip.run("""
allocs, frees = var("fake_allocs"), var("fake_frees")
fail_at = var("fake_fail_at")
L = ctypes.c_void_p()
allocs.value = 0
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0
n = allocs.value
lib.dbs_layer_destroy(L)
lib.dbs_layer_destroy(None)
assert frees.value == n
for k in range(n):
    allocs.value = frees.value = 0
    fail_at.value = k
    L = ctypes.c_void_p()
    assert lib.dbs_layer_create(None, ctypes.byref(L)) == 2 and not L.value
    fail_at.value = -1
    assert frees.value == allocs.value - 1
    assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0     # (the error does not stick)
    lib.dbs_layer_destroy(L)
""")
