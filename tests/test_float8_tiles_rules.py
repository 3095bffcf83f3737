"""That the sizes of the GPU tests of 8-bit products reach every tile, whole and in
parts (CPU only, kernels do not run)."""
import fake_hip
import test_edges_rules
import test_gpu_float8_tiles as tiles


def test_sizes_reach_all_tiles():
    fake_hip.run(test_edges_rules.CALLS + f"sizes, backward = {tiles.SIZES!r}, {tiles.BACKWARD!r}\n" + """
shapes = {"Li8ELi2ELi2E": "256x256", "Li4ELi1ELi4E": "128x128", "Li4ELi2ELi3E": "128x256", "Li2ELi1ELi3E": "64x128"}
units = {"256x256": 256, "128x128": 256, "128x256": 256, "64x128": 512}
def tiles_of(names):
    return [shapes[re.search("k_mul8.*?(Li[0-9]+ELi[0-9]+ELi[0-9]+E)E", v).group(1)] for v in names if "k_mul8" in v]
def one(t, n, m):
    names = linear(t, n, m, b8)[1]
    tile, = tiles_of(names)
    q, p = map(int, tile.split("x"))
    return tile, any("k_join" in v for v in names), -(-t // q) * -(-m // p) > units[tile]
# (the last tiles in parts, more tiles than run beside each other)
forms = {"256x256": [(False, False), (False, False), (False, True), (True, True)],
         "128x256": [(False, False), (False, False), (False, False), (True, True)],
         "128x128": [(False, False), (False, False), (True, False), (True, True)],
         "64x128": [(False, True), (True, True)]}
for tile, of in sizes.items():
    got = [one(*s) for s in of]
    assert got == [(tile, *f) for f in forms[tile]], (tile, got)
seen = set()
for t, n, m in backward:
    names = taken(lib.dbs_linear8_backward(L, 3, t, n, m, p, m, p, n, None, b8, p, n, p, n, p, p, room))[1]
    seen |= set(tiles_of(names))
assert {"256x256", "128x256", "128x128"} <= seen, seen
""")
