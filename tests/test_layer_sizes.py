"""Sizes at and past the dense layer operators' limits (CPU only)."""
import pytest
import torch

import fake_hip
from paper_2608_16308_amd import Checkpoint, DbsError, layer
from paper_2608_16308_amd._lib import DBS_ERR_UNSUPPORTED

META = torch.device("meta")
BF = torch.bfloat16


def test_sizes_that_do_not_fit_the_abi():
    """2^32 + 3 rows must not arrive as 3 (meta tensors have no memory)."""
    for shape in (((1 << 32) + 3, 1), (1, (1 << 32) + 3), ((1 << 31) + 1, 2), ((1 << 30) + 1, 1)):
        t = torch.empty(shape, dtype=BF, device=META)
        with pytest.raises(DbsError) as e:
            layer.check_rows(t, "x", BF, META, None, None)
        assert e.value.status == DBS_ERR_UNSUPPORTED
        c = Checkpoint(torch.empty(shape, dtype=torch.int8, device=META),
                       torch.empty((shape[0], -(-shape[1] // 32)), dtype=torch.uint8, device=META), BF)
        with pytest.raises(DbsError) as e:
            layer.check_checkpoint(torch, c, "c", BF, META, *shape)
        assert e.value.status == DBS_ERR_UNSUPPORTED
    for shape in ((1 << 30, 1), (1, 1 << 30)):
        layer.check_rows(torch.empty(shape, dtype=BF, device=META), "x", BF, META, None, None)

def test_launches_of_the_largest_sizes():
    """No launch has 2^32 threads or more, which the runtime refuses, at sizes
    that fit the device's memory (here there is none: kernels do not run)."""
    fake_hip.run("""
from paper_2608_16308_amd import _lib
L = ctypes.c_void_p()
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0
p = 1 << 20
H = lambda *v: ctypes.byref(_lib.Held(*v))
most, launches = var("fake_most_threads", ctypes.c_ulong), var("fake_launches")
def linear(t, n, m, keep=None):
    return lib.dbs_linear(L, 3, t, n, m, p, n, p, n, p, 2, None, 0, p, m, keep, None, 0)
def gated(t, n, m, keep=None):
    return lib.dbs_gated(L, 3, t, n, m, p, n, p, n, p, n, 2, p, m, keep, keep, None, 0)
def lback(t, n, m, dx=p, dw=p, db=p):
    return lib.dbs_linear_backward(L, 1, t, n, m, p, m, H(p, n, None, None), p, n, H(p, m, None, None), 2, dx, n, dw, n, db,
                                   p, 1 << 50)
def gback(t, n, m):
    return lib.dbs_gated_backward(L, 1, t, n, m, p, m, H(p, n, None, None), p, n, p, n, H(p, m, None, None), H(p, m, None, None),
                                  2, p, n, p, n, p, n, p, 1 << 50)
big = 1 << 30
for f, args in ((linear, (1, 8, big)), (gated, (1, 8, big)), (linear, (2, 8, big)), (gated, (2, 8, big)), (gated, (16, 256, big)),
                (linear, (17, 8, big)), (gated, (17, 1, big)), (gated, (17, 8, big)), (lback, (1, 8, big)), (gback, (1, 8, big)),
                (lback, (1, 1, big)), (gback, (2, big, 8)), (gback, (17, big, 1)), (lback, (17, big, 8)), (lback, (0, 0, big)),
                (linear, (big, 8, 17)), (gated, (big, 1, 1)), (gback, (big, 8, 1))):
    most.value = 0
    assert f(*args) == 0, (f.__name__, args, lib.dbs_last_error())
    assert 0 < most.value < 1 << 32, (f.__name__, args, most.value)
for name in ("dbs_pack", "dbs_unpack"):
    for rows, cols in ((big, 1), (1, big), (1 << 20, 1 << 16)):
        most.value = 0
        assert getattr(lib, name)(L, 3, rows, cols, *((p, cols, p, p) if name == "dbs_pack" else (p, p, p, cols))) == 0
        assert 0 < most.value < 1 << 32
""")
