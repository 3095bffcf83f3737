"""Which kernels norms with a small eps take (CPU only, kernels do not run): those that
take tiny rows 2^100 fold from eps below 2^-120 on, and only those."""
import fake_hip
import test_edges_rules


def test_eps():
    fake_hip.run(test_edges_rules.CALLS + """
import math
LEAST = 2.0 ** -120
below = float(np.nextafter(np.float32(LEAST), np.float32(0)))
def tiny(st):
    # the sixth parameter of k_edge_back is TINY, the fifth of k_edge
    names = [v for v in taken(st)[1] if "k_edge_total" not in v]
    flags = [re.findall("Lb([01])E", v)[-1] for v in names]
    assert len(flags) == 1, names
    return flags[0] == "1"
def norm(eps, kind=1):
    return R(_lib.NormDesc(kind, eps, p, None)) if eps is not None else None
for n in (8, 500, 4096, 8192, 16384):
    for kind in (1, 2):
        for eps, want in ((0.0, True), (below, True), (LEAST, False), (1e-6, False)):
            assert tiny(lib.dbs_norm(L, 3, 9, n, p, n, norm(eps, kind), p, n, None)) == want
            assert tiny(lib.dbs_norm_backward(L, 3, 9, n, p, n, p, n, norm(eps, kind), None, n, p, n, p, None, p, room)) == want
    for dt in (1, 3):
        for after, before, want in ((0.0, None, True), (None, 0.0, True), (1e-5, 0.0, True), (0.0, 1e-5, True), (1e-5, 1e-5, False), (1e-5, None, False),
                                    (None, 1e-5, False), (None, None, False)):
            a, b, h = norm(after), norm(before, 2), p if before is not None else None
            assert tiny(lib.dbs_join(L, dt, 9, n, p, n, p, n, a, b, None, 0, 1.0, None, p, n, h, n, None)) == want, (n, after, before)
            if n <= 8192:
                st = lib.dbs_join_backward(L, dt, 9, n, p, n, h, n, p, n, p, n, a, b, None, 0, 1.0, None, p, n, p, n, None, n, None, None, None, None, p, room)
                assert tiny(st) == want, (n, after, before)
""")
