"""Which kernels the norms, joins and 8-bit products take (CPU only, kernels do not
run), on both sides of the limits that were measured."""
import fake_hip

CALLS = """
import re
from paper_2608_16308_amd import _lib
L = ctypes.c_void_p()
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0
p, room = 1 << 20, 1 << 50
R = ctypes.byref
norm = lambda kind=1: R(_lib.NormDesc(kind, 1e-5, p, p))
b8 = R(_lib.Blocks(p, p))
fake.fake_launched.restype = ctypes.c_char_p
def taken(st):
    assert st == 0, lib.dbs_last_error()
    names = fake.fake_launched().decode().split()
    fake.fake_forget()
    return [re.search("[0-9](k_[a-z_0-9]+?)(I|E)", n).group(1) for n in names], names
def linear(t, n, m, x8=None):
    return taken(lib.dbs_linear8(L, 3, t, n, m, None if x8 else p, n, x8, b8, None, None, 0, p, m, p, room))
"""


def test_few_tokens():
    """Up to 16 tokens without tiles; up to 32 blocks of x for each wave packed on the way."""
    fake_hip.run(CALLS + """
size = ctypes.c_size_t()
for t, n, alone in ((1, 4096, True), (4, 4096, True), (5, 4096, False), (4, 1024, True), (5, 1024, False), (16, 1024, False), (2, 14336, True), (3, 14336, False),
                    (1, 32768, True), (1, 32769, False)):
    got = linear(t, n, 512)[0]
    assert got == (["k_rows8"] if alone else ["k_pack8_rows", "k_rows8"]), (t, n, got)
    assert linear(t, n, 512, b8)[0] == ["k_rows8"]
    assert lib.dbs_linear8_work(L, t, n, 512, ctypes.byref(size)) == 0 and (size.value == 0) == alone
assert linear(17, 1024, 512)[0][:2] == ["k_pack8_rows", "k_mul8"]
""")


def test_tiles():
    fake_hip.run(CALLS + """
def tile(t, n, m):
    names = linear(t, n, m, b8)[1]
    return {re.search("k_mul8.*?(Li[0-9]+ELi[0-9]+ELi[0-9]+E)E", v).group(1) for v in names if "k_mul8" in v}.pop()
big, square, flat, small = "Li8ELi2ELi2E", "Li4ELi1ELi4E", "Li4ELi2ELi3E", "Li2ELi1ELi3E"
for t, n, m, want in ((4096, 4096, 11008, big), (4096, 11008, 4096, big), (8192, 8192, 8192, big), (1531, 7001, 5003, flat), (2048, 4096, 4096, flat),
                      (1024, 11008, 4096, square), (777, 4096, 4096, square), (32, 4096, 11008, small), (320, 4096, 11008, small),
                      (512, 4096, 4096, small)):
    assert tile(t, n, m) == want, (t, n, m, tile(t, n, m))
""")


def test_rows_in_registers():
    fake_hip.run(CALLS + """
def fwd(n):
    return taken(lib.dbs_norm(L, 3, 9, n, p, n, norm(), p, n, None))[0]
assert fwd(16384) == ["k_edge"] and fwd(16385) == ["k_edge_long"]
assert fwd(8) == ["k_edge"] and fwd(7) == ["k_edge_long"]
def back(n):
    return taken(lib.dbs_norm_backward(L, 3, 9, n, p, n, p, n, norm(2), None, n, p, n, p, p, p, room))[0]
assert back(16384) == ["k_edge_back", "k_edge_total"] and back(16385) == ["k_edge_back_rows", "k_edge_back_strip", "k_edge_total"]
def jback(n):
    return taken(lib.dbs_join_backward(L, 3, 9, n, p, n, p, n, p, n, p, n, norm(), norm(), p, 0, 1.0, None, p, n, p, n, p, n, p, p, p, p, p, room))[0]
assert jback(8192) == ["k_edge_back", "k_edge_total"] and jback(8193) == ["k_edge_back_rows", "k_edge_back_strip", "k_edge_total"]
# the workspace that is asked for is enough on both sides
size = ctypes.c_size_t()
for n in (7, 8, 500, 900, 2048, 2049, 6144, 6145, 8192, 8193, 16384, 16385):
    for rows in (1, 9, 100000):
        assert lib.dbs_edge_work(L, rows, n, 2, ctypes.byref(size)) == 0
        taken(lib.dbs_norm_backward(L, 3, rows, n, p, n, p, n, norm(2), None, n, p, n, p, p, p, size.value))
        assert lib.dbs_edge_work(L, rows, n, 5, ctypes.byref(size)) == 0
        taken(lib.dbs_join_backward(L, 3, rows, n, p, n, p, n, p, n, p, n, norm(), norm(), p, 0, 1.0, None, p, n, p, n, p, n, p, p, p, p, p, size.value))
""")


def test_teams_of_the_gradients():
    """The waves that a join's gradients are compiled for, by the norms and the columns."""
    fake_hip.run(CALLS + """
def team(n, after, before):
    a, b = norm() if after else None, norm() if before else None
    names = taken(lib.dbs_join_backward(L, 3, 900, n, p, n, p if before else None, n, p, n, p, n, a, b, p, 0, 1.0, None, p, n, p, n, p, n,
                                        p if after else None, p if after else None, p if before else None, p if before else None, p, room))[1]
    return [tuple(map(int, re.search("k_edge_back.*?Li([0-9]+)ELi([0-9]+)E", v).groups())) for v in names if "k_edge_backI" in v][0]
for n, want in ((500, (1, 12)), (2048, (1, 12)), (2049, (1, 8)), (4096, (1, 8)), (4097, (1, 12)), (6144, (1, 12)), (6145, (2, 8)), (8192, (2, 8))):
    assert team(n, True, True) == want, (n, team(n, True, True))
for n, want in ((500, (1, 8)), (4096, (1, 8)), (4097, (1, 12)), (6145, (2, 8))):
    assert team(n, True, False) == want and team(n, False, True) == want, n
""")
