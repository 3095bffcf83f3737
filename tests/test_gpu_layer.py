"""Dense layer operators on the GPU against their definitions in 64 bits."""
import pytest
import torch

import layer_ref as ref
import paper_2608_16308_amd as dbs
from gpu_helpers import log

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]
# tokens, n_in, n_out: one of each, sizes around the tiles' and the groups'
# edges, single tokens and long sums
SIZES = [(1, 1, 1), (1, 64, 64), (1, 4096, 513), (2, 33, 31), (3, 257, 320), (8, 1024, 1000), (16, 72, 48), (17, 200, 96),
         (31, 8, 7), (64, 128, 256), (65, 4104, 130), (127, 63, 129), (130, 136, 264), (257, 512, 260), (300, 1001, 517),
         (520, 264, 776)]


@pytest.fixture(scope="module")
def ctx():
    return dbs.LayerContext()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, shape, dt, scale=1.0, pad=0, offset=0):
    """N(0, scale) in a buffer with rows `pad` longer that starts `offset`
    elements into it; what lies around is NaN."""
    rows, cols = shape
    buf = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=dt, device="cuda")
    v = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(shape, generator=g, device="cuda") * scale)
    return v


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear(ctx, size, dt):
    t, n, m = size
    g = gen(t * 7 + n * 3 + m)
    log(f"linear {size} {dt}")
    for i, kind in enumerate(ACTS):
        x, w = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5)
        bias = rnd(g, (1, m), dt)[0] if i % 2 else None
        res = rnd(g, (t, m), dt) if i % 3 else None
        y, ey, z, ez = ref.linear(x, w, bias, kind, res)
        ref.check(ctx.linear(x, w, bias=bias, act=kind, residual=res), y, ey, f"{size} {kind}")
        got, pre = ctx.linear(x, w, bias=bias, act=kind, residual=res, save="full")
        ref.check(got, y, ey, f"{size} {kind} saving")
        ref.check(pre, z, ez, f"{size} {kind} pre")
        got8, pre8 = ctx.linear(x, w, bias=bias, act=kind, residual=res, save="8bit")
        assert torch.equal(got8, got)
        codes, exps = ref.pack(pre.cpu())
        assert torch.equal(pre8.codes.cpu(), codes) and torch.equal(pre8.exponents.cpu(), exps)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated(ctx, size, dt):
    t, n, m = size
    g = gen(t * 5 + n * 11 + m)
    log(f"gated {size} {dt}")
    for kind in ACTS:
        x, wg, wu = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5)
        h, eh, gate, eg, up, eu = ref.gated(x, wg, wu, kind)
        ref.check(ctx.gated(x, wg, wu, act=kind), h, eh, f"{size} {kind}")
        got, kg, ku = ctx.gated(x, wg, wu, act=kind, save="full")
        ref.check(got, h, eh, f"{size} {kind} saving")
        ref.check(kg, gate, eg, f"{size} {kind} gate")
        ref.check(ku, up, eu, f"{size} {kind} up")
        got8, g8, u8 = ctx.gated(x, wg, wu, act=kind, save="8bit")
        assert torch.equal(got8, got)
        for full, held in ((kg, g8), (ku, u8)):
            codes, exps = ref.pack(full.cpu())
            assert torch.equal(held.codes.cpu(), codes) and torch.equal(held.exponents.cpu(), exps)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_backward(ctx, size, dt):
    t, n, m = size
    g = gen(t * 3 + n * 5 + m)
    log(f"linear backward {size} {dt}")
    for i, kind in enumerate(ACTS):
        x, w, dy, pre = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (t, m), dt), rnd(g, (t, m), dt)
        for held in ("full", "8bit"):
            hx, hp = (x, pre) if held == "full" else (ctx.pack(x), ctx.pack(pre))
            vx, vp = (x, pre) if held == "full" else (ctx.unpack(hx), ctx.unpack(hp))
            want = ref.linear_backward(dy, vx.double(), w, vp.double(), kind)
            got = ctx.linear_backward(dy, hx, w, pre=None if kind == "none" else hp, act=kind, bias=True)
            for name, v in zip(("dx", "dw", "db"), got):
                ref.check(v, *want[name], f"{size} {kind} {held} {name}")
    dx, dw, db = ctx.linear_backward(dy, x, w, pre=pre, act=kind, need_dx=False)
    assert dx is None and db is None and torch.equal(dw, ctx.linear_backward(dy, x, w, pre=pre, act=kind)[1])
    dx, dw, db = ctx.linear_backward(dy, None, w, pre=pre, act=kind, need_dw=False, bias=True)
    assert dw is None and torch.equal(dx, ctx.linear_backward(dy, x, w, pre=pre, act=kind)[0])


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated_backward(ctx, size, dt):
    t, n, m = size
    g = gen(t * 13 + n * 5 + m)
    log(f"gated backward {size} {dt}")
    for kind in ACTS:
        x, wg, wu = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5)
        dh, gate, up = rnd(g, (t, m), dt), rnd(g, (t, m), dt), rnd(g, (t, m), dt)
        for held in ("full", "8bit"):
            hs = (x, gate, up) if held == "full" else tuple(ctx.pack(v) for v in (x, gate, up))
            vx, vg, vu = (v if held == "full" else ctx.unpack(v) for v in hs)
            want = ref.gated_backward(dh, vx.double(), wg, wu, vg.double(), vu.double(), kind)
            got = ctx.gated_backward(dh, hs[0], wg, wu, hs[1], hs[2], act=kind)
            for name, v in zip(("dx", "dw_gate", "dw_up"), got):
                ref.check(v, *want[name], f"{size} {kind} {held} {name}")
    dx, a, b = ctx.gated_backward(dh, None, wg, wu, gate, up, act=kind, need_dw=False)
    assert a is None and b is None and torch.equal(dx, ctx.gated_backward(dh, x, wg, wu, gate, up, act=kind)[0])


# rows in wider buffers, bases off their alignment, mixed
@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 0), (8, 0), (64, 8), (5, 3), (8, 4)])
@pytest.mark.parametrize("size", [(1, 256, 192), (5, 264, 136), (40, 250, 70), (200, 256, 256), (150, 129, 77)], ids=str)
def test_strides_and_alignment(ctx, size, pad, offset, dt):
    t, n, m = size
    g = gen(t + n + m + pad * 17 + offset)
    log(f"strides {size} pad {pad} offset {offset} {dt}")
    at = dict(pad=pad, offset=offset)
    x, w, wu = rnd(g, (t, n), dt, **at), rnd(g, (m, n), dt, n ** -0.5, **at), rnd(g, (m, n), dt, n ** -0.5)
    res, bias = rnd(g, (t, m), dt, **at), rnd(g, (1, m), dt, offset=offset)[0]
    y = rnd(g, (t, m), dt, **at)
    want, bound, _, _ = ref.linear(x, w, bias, "silu", res)
    out = ctx.linear(x, w, bias=bias, act="silu", residual=res, y=y)
    assert out.data_ptr() == y.data_ptr()
    ref.check(y, want, bound, "linear into y")
    ref.check(ctx.linear(x, w, bias=bias, act="silu", residual=res, y=res), want, bound, "linear onto its residual")
    h = rnd(g, (t, m), dt, **at)
    want, bound = ref.gated(x, w, wu, "gelu")[:2]
    ctx.gated(x, w, wu, act="gelu", h=h)
    ref.check(h, want, bound, "gated into h")
    # nothing beside the rows is written
    if pad:
        for v in (y, h):
            full = torch.as_strided(v, (t, pad), (v.stride(0), 1), v.storage_offset() + m)
            assert full.isnan().all()
    dy, pre = rnd(g, (t, m), dt, **at), rnd(g, (t, m), dt, **at)
    want = ref.linear_backward(dy, x.double(), w, pre.double(), "gelu_tanh")
    for name, v in zip(("dx", "dw", "db"), ctx.linear_backward(dy, x, w, pre=pre, act="gelu_tanh", bias=True)):
        ref.check(v, *want[name], name)
    want = ref.linear_backward(dy, x.double(), w, None, "none")
    for name, v in zip(("dx", "dw", "db"), ctx.linear_backward(dy, x, w, bias=True)):
        ref.check(v, *want[name], name + " without activation")
    want = ref.gated_backward(dy, x.double(), w, wu, pre.double(), h.double(), "silu")
    for name, v in zip(("dx", "dw_gate", "dw_up"), ctx.gated_backward(dy, x, w, wu, pre, h)):
        ref.check(v, *want[name], name)


# tokens on either side of each kernel's range, sums of a turn, of several and
# of a ragged one, rows that are shorter than a load
@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("n", [7, 8, 9, 255, 256, 264, 2049, 4100])
@pytest.mark.parametrize("t", [1, 2, 5, 15, 16, 17, 33, 64, 65])
def test_few_tokens(ctx, t, n, dt):
    m = 70
    g = gen(t * 31 + n)
    log(f"few tokens {t} {n} {dt}")
    x, w, wu = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5)
    bias, res = rnd(g, (1, m), dt)[0], rnd(g, (t, m), dt)
    y, ey, z, ez = ref.linear(x, w, bias, "silu", res)
    got, pre = ctx.linear(x, w, bias=bias, act="silu", residual=res, save="full")
    ref.check(got, y, ey, "linear")
    ref.check(pre, z, ez, "pre")
    got8, pre8 = ctx.linear(x, w, bias=bias, act="silu", residual=res, save="8bit")
    assert torch.equal(got8, got) and torch.equal(pre8.codes.cpu(), ref.pack(pre.cpu())[0])
    h, eh = ref.gated(x, w, wu, "gelu")[:2]
    got, gate, up = ctx.gated(x, w, wu, act="gelu", save="full")
    ref.check(got, h, eh, "gated")
    got8, g8, u8 = ctx.gated(x, w, wu, act="gelu", save="8bit")
    assert torch.equal(got8, got)
    for full, held in ((gate, g8), (up, u8)):
        codes, exps = ref.pack(full.cpu())
        assert torch.equal(held.codes.cpu(), codes) and torch.equal(held.exponents.cpu(), exps)
    if t == 1:
        assert torch.equal(ctx.linear(x[0], w, bias=bias, act="silu", residual=res[0]), ctx.linear(x, w, bias=bias, act="silu", residual=res)[0])
        assert torch.equal(ctx.gated(x[0], w, wu, act="gelu"), got[0])


# rounds of whole tiles with a rest in parts, several rows and columns of tiles,
# operands in whole chunks, in odd places and copied from there
@pytest.mark.parametrize("size", [(1024, 4096, 1032), (520, 2056, 4104), (300, 4099, 1500), (700, 3001, 2003), (90, 8200, 600)], ids=str)
def test_larger_products(ctx, size):
    t, n, m = size
    dt = torch.bfloat16
    g = gen(sum(size))
    log(f"larger {size}")
    x, w, wu, dy = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (t, m), dt)
    res = rnd(g, (t, m), dt)
    y, ey, _, _ = ref.linear(x, w, None, "gelu_tanh", res)
    ref.check(ctx.linear(x, w, act="gelu_tanh", residual=res), y, ey, "linear")
    h, eh, gate, eg, up, eu = ref.gated(x, w, wu, "silu")
    got, kg, ku = ctx.gated(x, w, wu, save="full")
    ref.check(got, h, eh, "gated")
    ref.check(kg, gate, eg, "gate")
    ref.check(ku, up, eu, "up")
    want = ref.gated_backward(dy, x.double(), w, wu, kg.double(), ku.double(), "silu")
    for name, v in zip(("dx", "dw_gate", "dw_up"), ctx.gated_backward(dy, x, w, wu, kg, ku)):
        ref.check(v, *want[name], name)
    want = ref.linear_backward(dy, x.double(), w, None, "none")
    for name, v in zip(("dx", "dw", "db"), ctx.linear_backward(dy, x, w, bias=True)):
        ref.check(v, *want[name], name)


def test_without_workspace(ctx):
    """Operands in odd places, with the copies that a workspace allows and without."""
    import ctypes
    from paper_2608_16308_amd import _lib
    dt, (t, n, m) = torch.float16, (2000, 3001, 2003)
    g = gen(6)
    x, w, y = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), torch.empty((t, m), dtype=dt, device="cuda")
    want, bound, _, _ = ref.linear(x, w, None, "none", None)
    size = ctypes.c_size_t()
    _lib.check(dbs.lib().dbs_forward_work(ctx._h, 0, t, n, m, ctypes.byref(size)))
    assert size.value >= 2 * (t * n + m * n)
    work = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    for at, room in ((work.data_ptr(), size.value), (work.data_ptr(), 1024), (None, 0)):
        y.fill_(float("nan"))
        _lib.check(dbs.lib().dbs_linear(ctx._h, _lib.DBS_F16, t, n, m, x.data_ptr(), n, w.data_ptr(), n, None, 0, None, 0,
                                        y.data_ptr(), m, None, at, room))
        ref.check(y, want, bound, f"{room} bytes")


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_empty_sizes(ctx, dt):
    z = lambda *s: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    one = lambda *s: torch.ones(s, dtype=dt, device="cuda")  # noqa: E731
    assert ctx.linear(z(0, 8), z(5, 8)).shape == (0, 5) and ctx.linear(z(3, 8), z(0, 8)).shape == (3, 0)
    assert ctx.gated(z(0, 8), z(5, 8), z(5, 8)).shape == (0, 5)
    # an empty sum: the bias, the activation of it, the residual
    y, pre = ctx.linear(z(3, 0), z(40, 0), bias=one(40), act="relu", residual=one(3, 40), save="8bit")
    assert torch.equal(y, 2 * one(3, 40)) and torch.equal(ctx.unpack(pre), one(3, 40))
    assert torch.equal(ctx.linear(z(0), z(40, 0)), z(40)) and torch.equal(ctx.gated(z(3, 0), z(40, 0), z(40, 0)), z(3, 40))
    # no token: the weights' gradients are zero
    dx, dw, db = ctx.linear_backward(z(0, 6), z(0, 9), z(6, 9), pre=z(0, 6), act="silu", bias=True)
    assert dx.shape == (0, 9) and torch.equal(dw, z(6, 9)) and torch.equal(db, z(6))
    dx, a, b = ctx.gated_backward(z(0, 6), z(0, 9), z(6, 9), z(6, 9), z(0, 6), z(0, 6))
    assert dx.shape == (0, 9) and torch.equal(a, z(6, 9)) and torch.equal(b, z(6, 9))
    dx, dw, db = ctx.linear_backward(z(4, 0), one(4, 9), z(0, 9), bias=True)
    assert torch.equal(dx, z(4, 9)) and dw.shape == (0, 9) and db.shape == (0,)
    c = ctx.pack(z(0, 7))
    assert c.codes.shape == (0, 7) and ctx.unpack(c).shape == (0, 7) and ctx.unpack(ctx.pack(z(4, 0))).shape == (4, 0)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 100, 70), (8, 264, 72), (70, 300, 140), (260, 512, 264)], ids=str)
def test_not_finite(ctx, size, dt):
    """NaN and infinities reach what depends on them and nothing else."""
    t, n, m = size
    g = gen(99)
    x, w, wu = rnd(g, size[:2], dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5)
    x[t - 1, n - 1] = float("nan")
    w[m - 1, 0] = float("inf")
    y, ey, z, ez = ref.linear(x, w, None, "none", None)
    assert bool(y[:t - 1, :m - 1].isfinite().all())
    got, pre = ctx.linear(x, w, save="full")
    ref.check(got, y, ey, "linear")
    ref.check(pre, z, ez, "pre")
    _, held = ctx.linear(x, w, save="8bit")
    codes, exps = ref.pack(pre.cpu())
    assert torch.equal(held.codes.cpu(), codes) and torch.equal(held.exponents.cpu(), exps)
    w[m - 1, 0] = 0
    h, eh = ref.gated(x, w, wu, "silu")[:2]
    ref.check(ctx.gated(x, w, wu), h, eh, "gated")
    dy = rnd(g, (t, m), dt)
    pre = rnd(g, (t, m), dt)
    pre[0, m - 1] = float("nan")
    for hx, hp in ((x, pre), (ctx.pack(x), ctx.pack(pre))):
        vx, vp = (v if isinstance(v, torch.Tensor) else ctx.unpack(v) for v in (hx, hp))
        want = ref.linear_backward(dy, vx.double(), w, vp.double(), "silu")
        for name, v in zip(("dx", "dw", "db"), ctx.linear_backward(dy, hx, w, pre=hp, act="silu", bias=True)):
            ref.check(v, *want[name], name)


@pytest.mark.parametrize("kind", ACTS)
def test_activation_tails(ctx, kind):
    """Arguments over the whole range, through a sum of one term."""
    for dt in TYPES:
        z = torch.cat([torch.linspace(-30, 30, 4001), torch.tensor([0.0, 1e4, -1e4, 6e4, -6e4])]).to(dt).cuda()
        x, w = z[:, None].contiguous(), torch.ones((1, 1), dtype=dt, device="cuda")
        y, ey, _, _ = ref.linear(x, w, None, kind, None)
        ref.check(ctx.linear(x, w, act=kind), y, ey, f"{kind} {dt}")
        dy = torch.ones_like(x)
        want = ref.linear_backward(dy, x.double(), w, x.double(), kind)
        dx, _, _ = ctx.linear_backward(dy, x, w, pre=None if kind == "none" else x, act=kind)
        ref.check(dx, *want["dx"], f"slope {kind} {dt}")


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "none"])
def test_gradients_against_differences(ctx, kind):
    """Along random directions, against central differences of the definition."""
    dt, (t, n, m) = torch.float16, (37, 90, 75)
    g = gen(5)
    x, w, wu = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5)
    b, dy = rnd(g, (1, m), dt)[0], rnd(g, (t, m), dt)
    X, W, WU, B, D = (v.double() for v in (x, w, wu, b, dy))
    h = 2.0 ** -14

    def along(loss, args, grads, bounds, kept):
        for i, (grad, bound) in enumerate(zip(grads, bounds)):
            v = torch.randn(args[i].shape, generator=g, device="cuda", dtype=torch.float64)
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + h * v, args[i] - h * v
            diff = float(loss(*up) - loss(*down)) / (2 * h)
            got = float((grad.double() * v).sum())
            # the bound of the gradient, what rounding the kept projections
            # changes it by, and the differences' own error (third derivatives
            # of at most 3 along v; sums of doubles)
            room = float((bound * v.abs()).sum()) + kept[i](v) + h * h * 3 * float((D.abs().sum() * (v.abs().max() ** 3 + 1)) * n ** 1.5) + 1e-6
            assert abs(got - diff) <= room, (kind, i, got, diff, room)

    _, pre = ctx.linear(x, w, bias=b, act=kind, save="full")
    want = ref.linear_backward(dy, X, w, pre.double(), kind)
    got = ctx.linear_backward(dy, x, w, pre=None if kind == "none" else pre, act=kind, bias=True)
    # a slope changes by at most 1.2 of the rounding of its argument (second
    # derivatives of these activations are below 1.2)
    ez = 1.2 * ref.linear(x, w, b, kind, None)[3] * D.abs()
    along(lambda a, c, d: (D * ref.act(a @ c.T + d, kind)).sum(), (X, W, B), got, [want[k][1] for k in ("dx", "dw", "db")],
          [lambda v: float((ez * (v.abs() @ W.abs().T)).sum()), lambda v: float((ez * (X.abs() @ v.abs().T)).sum()),
           lambda v: float((ez * v.abs()).sum())])
    _, gate, up = ctx.gated(x, w, wu, act=kind, save="full")
    want = ref.gated_backward(dy, X, w, wu, gate.double(), up.double(), kind)
    got = ctx.gated_backward(dy, x, w, wu, gate, up, act=kind)
    _, _, G, eg, U, eu = ref.gated(x, w, wu, kind)
    e1 = D.abs() * (1.2 * eg * (U.abs() + eu) + 1.2 * eu)   # of dg
    e2 = D.abs() * 1.2 * eg                                 # of du
    along(lambda a, c, d: (D * ref.act(a @ c.T, kind) * (a @ d.T)).sum(), (X, W, WU), got,
          [want[k][1] for k in ("dx", "dw_gate", "dw_up")],
          [lambda v: float((e1 * (v.abs() @ W.abs().T) + e2 * (v.abs() @ WU.abs().T)).sum()),
           lambda v: float((e1 * (X.abs() @ v.abs().T)).sum()), lambda v: float((e2 * (X.abs() @ v.abs().T)).sum())])


# ---------------------------------------------------------------------------
# checkpoints
# ---------------------------------------------------------------------------
def ck_values(g, rows, cols, dt):
    """Magnitudes over the type's whole range, zeros, group edges, largest
    numbers, values that are not finite."""
    span = 250 if dt == torch.bfloat16 else 38
    least = -134 if dt == torch.bfloat16 else -25
    e = torch.randint(0, span, (rows, 1), generator=g, device="cuda").double() + least
    v = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.float64) * 2.0 ** e
    x = v.clamp(-ref.MAX[dt], ref.MAX[dt]).to(dt)
    if rows > 6:
        x[0] = 0
        x[1, :] = ref.MAX[dt]
        x[2, cols // 2] = float("inf")
        x[3, 0] = float("nan")
        x[4] = float("-inf")
        x[5] = 127 * 2.0 ** -9
        x[6] = 127.5 * 2.0 ** -9
    return x


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (9, 31), (40, 33), (64, 96), (33, 257), (7, 4099), (1000, 64)])
def test_checkpoint_codes(ctx, rows, cols, dt):
    x = ck_values(gen(rows * cols), rows, cols, dt)
    for v in (x, torch.nn.functional.pad(x, (1, 4), value=float("inf"))[:, 1:1 + cols]):
        c = ctx.pack(v)
        codes, exps = ref.pack(x.cpu())
        assert torch.equal(c.codes.cpu(), codes) and torch.equal(c.exponents.cpu(), exps)
        got, want = ctx.unpack(c).cpu().double(), ref.unpack(codes, exps, dt)
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    # a second trip changes nothing
    back = ctx.unpack(c)
    again = ctx.unpack(ctx.pack(back))
    assert torch.equal(torch.nan_to_num(back, nan=1.0), torch.nan_to_num(again, nan=1.0))
    y = torch.full((rows, cols + 3), 7.0, dtype=dt, device="cuda")
    ctx.unpack(c, y=y[:, :cols])
    assert torch.equal(torch.nan_to_num(y[:, :cols]), torch.nan_to_num(back)) and bool((y[:, cols:] == 7).all())


# ---------------------------------------------------------------------------
# streams, graphs, repeated calls
# ---------------------------------------------------------------------------
def test_other_stream():
    """A context on a stream of its own, called while another is current."""
    side = torch.cuda.Stream()
    ctx = dbs.LayerContext(stream=side)
    g = gen(3)
    dt = torch.bfloat16
    x, w, wu = rnd(g, (200, 512), dt), rnd(g, (300, 512), dt, 0.04), rnd(g, (300, 512), dt, 0.04)
    side.wait_stream(torch.cuda.current_stream())
    h, gate, up = ctx.gated(x, w, wu, save="8bit")
    dx, a, b = ctx.gated_backward(h, ctx.pack(x), w, wu, gate, up)
    keep = x.clone()
    del x
    side.synchronize()
    want, bound = ref.gated(keep, w, wu, "silu")[:2]
    ref.check(h, want, bound, "gated on a side stream")
    here = dbs.LayerContext()
    for p, q in zip((dx, a, b), here.gated_backward(h, here.pack(keep), w, wu, gate, up)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("size", [(1, 1024, 512), (8, 512, 264), (40, 2048, 256), (300, 512, 512)], ids=str)
def test_graph_replay(size):
    """Captured calls replay on new inputs, between eager work."""
    t, n, m = size
    dt = torch.float16
    g = gen(8)
    x, w, wu, down = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (n, m), dt, m ** -0.5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ctx = dbs.LayerContext()
        ctx.linear(ctx.gated(x, w, wu), down, residual=x)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            h = ctx.gated(x, w, wu)
            y = ctx.linear(h, down, residual=x)
            dx, dw, _ = ctx.linear_backward(y, h, down)
    torch.cuda.synchronize()
    eager = dbs.LayerContext()
    for i in range(4):
        x.copy_(torch.randn((t, n), generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        h2 = eager.gated(x, w, wu)
        y2 = eager.linear(h2, down, residual=x)
        dx2, dw2, _ = eager.linear_backward(y2, h2, down)
        torch.cuda.synchronize()
        for p, q in ((h, h2), (y, y2), (dx, dx2), (dw, dw2)):
            assert torch.equal(p, q), i


def test_same_bits_every_time(ctx):
    g = gen(21)
    dt = torch.bfloat16
    for t, n, m in ((1, 3000, 500), (24, 4096, 512), (100, 4096, 264), (700, 640, 648)):
        x, w, wu, dy = rnd(g, (t, n), dt), rnd(g, (m, n), dt), rnd(g, (m, n), dt), rnd(g, (t, m), dt)
        first = None
        for _ in range(5):
            out = [ctx.linear(x, w), ctx.gated(x, w, wu), *ctx.linear_backward(dy, x, w, bias=True)]
            first = first or out
            assert all(torch.equal(p, q) for p, q in zip(first, out))


def test_rows_past_32_bits(ctx):
    """A tensor whose last rows start beyond 2^32 bytes."""
    dt = torch.float16
    rows, ld = 5, (1 << 30) + 64
    big = torch.zeros(rows * ld, dtype=dt, device="cuda")
    x = big.as_strided((rows, 96), (ld, 1))
    g = gen(4)
    x.copy_(torch.randn((rows, 96), generator=g, device="cuda"))
    w = rnd(g, (80, 96), dt, 0.1)
    y, ey, _, _ = ref.linear(x, w, None, "none", None)
    ref.check(ctx.linear(x, w), y, ey, "far rows")
    dy = rnd(g, (rows, 80), dt)
    want = ref.linear_backward(dy, x.double(), w, None, "none")
    ref.check(ctx.linear_backward(dy, x, w)[1], *want["dw"], "dw of far rows")
    c = ctx.pack(x)
    assert torch.equal(c.codes.cpu(), ref.pack(x.cpu().contiguous())[0])


def test_gradients_of_rows_far_apart(ctx):
    """Without an activation dy is multiplied as it is, whatever its rows' distance."""
    dt = torch.bfloat16
    g = gen(23)
    for t, m, ld in ((1, (1 << 21) + 8, None), (2, 80, (1 << 21) + 8)):
        x, w = rnd(g, (t, 8), dt), rnd(g, (m, 8), dt)
        buf = torch.zeros((t, ld or m), dtype=dt, device="cuda")
        dy = buf[:, :m]
        dy.copy_(torch.randn((t, m), generator=g, device="cuda"))
        want = ref.linear_backward(dy, x.double(), w, None, "none")
        for name, v in zip(("dx", "dw"), ctx.linear_backward(dy, x, w)):
            ref.check(v, *want[name], f"{t}x{m} rows of {ld or m} {name}")
