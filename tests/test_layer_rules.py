"""Which kernels a call of the dense layers takes (CPU only, kernels do not run),
on both sides of the limits that were measured."""
import fake_hip

CALLS = """
import re
from paper_2608_16308_amd import _lib
L = ctypes.c_void_p()
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0
p = 1 << 20
H = lambda *v: ctypes.byref(_lib.Held(*v))
fake.fake_launched.restype = ctypes.c_char_p
def taken(st):
    assert st == 0, lib.dbs_last_error()
    names = fake.fake_launched().decode().split()
    fake.fake_forget()
    return [re.search("k_[a-z_]+", n).group(0) for n in names if not "k_join" in n], names
def forward(t, n, m):
    size = ctypes.c_size_t()
    assert lib.dbs_forward_work(L, 0, t, n, m, ctypes.byref(size)) == 0
    return taken(lib.dbs_linear(L, 1, t, n, m, p, n, p, n, None, 0, None, 0, p, m, None, p if size.value else None, size.value))
def backward(gated, t, n, m, dx, dw):
    size = ctypes.c_size_t()
    assert lib.dbs_backward_work(L, gated, 0, t, n, m, 0, 0, 0, ctypes.byref(size)) == 0
    x, dx, dw, v = H(p, n, None, None), p if dx else None, p if dw else None, H(p, m, None, None)
    if gated:
        return taken(lib.dbs_gated_backward(L, 3, t, n, m, p, m, x, p, n, p, n, v, v, 0, dx, n, dw, n, dw, n, p, size.value))
    return taken(lib.dbs_linear_backward(L, 3, t, n, m, p, m, x, p, n, None, 0, dx, n, dw, n, None, p, size.value))
"""


def test_copies_of_odd_operands():
    """Into whole chunks where that is faster."""
    fake_hip.run(CALLS + """
for size in ((777, 1111, 2003), (1531, 1111, 2003), (2000, 2001, 2003)):
    assert forward(*size)[0] == ["k_tile"], size
for size in ((1531, 7001, 5003), (4096, 4097, 4096), (4096, 4097, 11007)):
    assert [k for k in forward(*size)[0] if k != "k_align"] == ["k_block"], size
for size in ((777, 1111, 2003), (2000, 3001, 2003), (4096, 4097, 4099)):
    for gated in (0, 1):
        for dx, dw in ((1, 0), (0, 1), (1, 1)):
            kernels = backward(gated, *size, dx, dw)[0]
            assert "k_tile" not in kernels and kernels.count("k_align") == dx * (1 + gated) + dw, (size, gated, kernels)
for dx, dw in ((1, 0), (0, 1)):
    assert "k_align" not in backward(0, 100, 1111, 2003, dx, dw)[0]
""")


def test_tiles_of_the_backward_products():
    """128x128 with four stages is a tile of the forward products."""
    fake_hip.run(CALLS + """
def tile(names):
    return {re.search("k_block.*?(Li[0-9]+ELi[0-9]+ELi[0-9]+ELi[0-9]+E)E", n).group(1) for n in names if "k_block" in n}
big, medium, small = "Li2ELi4ELi8ELi2E", "Li4ELi2ELi2ELi4E", "Li2ELi2ELi2ELi3E"
seen = set()
for t in (24, 40, 128, 320, 776, 1024, 2048, 4096):
    for n, m in ((1112, 2008), (2048, 2048), (4096, 1024), (1024, 4096), (4096, 4096), (4096, 11008), (11008, 4096)):
        for gated in (0, 1):
            got = tile(backward(gated, t, n, m, 1, 1)[1])
            assert got <= {big, small}, (t, n, m, got)
            seen |= got
        seen |= tile(forward(t, n, m)[1])
assert seen == {big, medium, small}, seen
for t, n, m, dx, dw, want in ((1024, 4096, 4096, 1, 0, big), (320, 2048, 2048, 1, 0, small), (320, 2048, 2048, 0, 1, small),
                              (4096, 4096, 11008, 1, 1, big)):
    assert tile(backward(0, t, n, m, dx, dw)[1]) == {want}, (t, n, m)
""")
