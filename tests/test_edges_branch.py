"""A join's gradients read the branch only where a gate or a norm after it needs it:
elsewhere neither its address nor its stride is checked, so the kernels do not get it
(CPU only, kernels do not run)."""
import fake_hip

CALLS = """
from paper_2608_16308_amd import _lib
L = ctypes.c_void_p()
assert lib.dbs_layer_create(None, ctypes.byref(L)) == 0
p, room = 1 << 20, 1 << 50
norm = ctypes.byref(_lib.NormDesc(1, 1e-5, p, None))
first = (ctypes.c_uint64 * 8 * 16).in_dll(fake, "fake_first")
keep, kept = var("fake_keep"), var("fake_kept")
keep.value = 32  # ds, dh, branch, stream
def branches(n, branch, ldb, after=None, before=None, gate=None):
    kept.value = 0
    st = lib.dbs_join_backward(L, 3, 5, n, p, n, p + 64 if before else None, n, branch, ldb, p + 128, n, after, before, gate, 0, 1.0, None, p, n,
                               p, n, None, n, None, None, None, None, p, room)
    # (the launches of one call; without sums no others follow)
    got = [tuple(first[i]) for i in range(kept.value)]
    assert all(g[0] == p for g in got)
    return st, {g[2] for g in got}
"""


def test_a_branch_that_is_not_needed_is_not_handed_on():
    fake_hip.run(CALLS + """
for n in (7, 64, 4096, 8192, 8193, 20000):  # rows in registers, and longer and shorter ones
    for before in (None, norm):
        for branch, ldb in ((p + 1, -(1 << 40)), (p, n), (p, 0), (None, 0)):
            assert branches(n, branch, ldb, before=before) == (0, {0}), (n, before, branch)
        for need in (dict(after=norm), dict(gate=p)):
            assert branches(n, p, n, before=before, **need) == (0, {p})
            for branch, ldb in ((p + 1, n), (p, n - 1), (p, -(1 << 40)), (None, n)):
                st, got = branches(n, branch, ldb, before=before, **need)
                assert st == 1 and not got, (n, need, branch)
""")
