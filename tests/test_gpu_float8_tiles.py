"""Products in 8-bit floating point of every tile, whole and in parts along k, on the GPU
against 64 bits."""
import pytest
import torch

import float8_ref as ref
import layer_ref
import paper_2608_16308_amd as dbs
from gpu_helpers import log

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
# tokens, n_in, n_out by the tile that the rule takes, ragged in all three: tiles that
# are all whole, in one round and in more; a last round in parts, alone and behind whole ones
SIZES = {
    "256x256": [(2111, 110, 5186), (1101, 1100, 9221), (2885, 1144, 8601), (2227, 1638, 7361)],
    "128x256": [(521, 100, 7787), (518, 1113, 7311), (1531, 7001, 5003), (1241, 1320, 6636)],
    "128x128": [(193, 101, 9050), (134, 1108, 11140), (844, 4814, 519), (481, 2068, 8381)],
    "64x128": [(1410, 1109, 5391), (517, 2122, 7209)],
}
# tokens, n_in, n_out whose gradients' products take the large tiles
BACKWARD = [(1101, 9221, 1100), (518, 7311, 1113), (481, 8381, 2068)]


@pytest.fixture(scope="module")
def ctx():
    return dbs.LayerContext()


def rnd(g, shape, dt, scale=1.0, pad=0):
    """N(0, scale) in rows `pad` longer; what lies around is NaN."""
    rows, cols = shape
    v = torch.full((rows + 2, cols + pad), float("nan"), dtype=dt, device="cuda")[1:-1, :cols]
    return v.copy_(torch.randn(shape, generator=g, device="cuda") * scale)


def product(q, p, dt, bias=None, residual=None):
    """float8_ref.product, computed on the GPU in 64 bits."""
    q, p = q.cuda(), p.cuda()
    eight = lambda v: torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 8)).unflatten(1, (-1, 8)).amax(2)  # noqa: E731
    y = q @ p.T.contiguous()
    e = 2 * layer_ref.sum_err(q.shape[1], q.abs() @ p.abs().T.contiguous()) + 7 * 2.0 ** -13 * (eight(q) @ eight(p).T.contiguous())
    for more in (bias, residual):
        if more is not None:
            y = y + more.double()
            e = e + 2.0 ** -24 * (y.abs() + e)
    return y, layer_ref.rounded(y, e, dt)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [s for v in SIZES.values() for s in v], ids=str)
def test_linear(ctx, size, dt):
    t, n, m = size
    g = torch.Generator(device="cuda")
    g.manual_seed(t + n + m)
    log(f"linear8 {size} {dt}")
    x, w = rnd(g, (t, n), dt, pad=3), rnd(g, (m, n), dt, n ** -0.5)
    bias, res = rnd(g, (1, m), dt)[0], rnd(g, (t, m), dt, pad=5)
    w8, x8 = ctx.pack8(w, block="tile"), ctx.pack8(x)
    vx, vw = ref.values(x8), ref.values(w8)
    layer_ref.check(ctx.linear8(x8, w8), *product(vx, vw, dt), f"{size}")
    y = ctx.linear8(x8, w8, bias=bias, residual=res)
    layer_ref.check(y, *product(vx, vw, dt, bias, res), f"{size} with bias and residual")
    buf = torch.full((t + 2, m + 16), 7.0, dtype=dt, device="cuda")
    around = torch.ones_like(buf, dtype=torch.bool)
    around[1:t + 1, 8:8 + m] = False
    for _ in range(3):  # (the same bits every time)
        assert torch.equal(ctx.linear8(x, w8, bias=bias, residual=res, y=buf[1:t + 1, 8:8 + m]), y)
    assert bool((buf[around] == 7.0).all())


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", BACKWARD, ids=str)
def test_backward(ctx, size, dt):
    t, n, m = size
    g = torch.Generator(device="cuda")
    g.manual_seed(t + n + m)
    log(f"linear8 backward {size} {dt}")
    x, w, dy = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (t, m), dt, pad=3)
    w8 = ctx.pack8(w, block="tile")
    dx, dw, db = ctx.linear8_backward(dy, x, w8, bias=True)
    vdy, vdt = ref.values(ctx.pack8(dy)), ref.values(ctx.pack8(dy, across=True))
    layer_ref.check(dx, *product(vdy, ref.values(w8).T, dt), f"{size} dx")
    layer_ref.check(dw, *product(vdt, ref.values(ctx.pack8(x, across=True)), dt), f"{size} dw")
    s = dy.double().sum(0)
    layer_ref.check(db, s, layer_ref.rounded(s, layer_ref.sum_err(t, dy.double().abs().sum(0)), dt), f"{size} db")
