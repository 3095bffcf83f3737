"""Blocks of 8-bit floating point and their products on the GPU against exact arithmetic."""
import pytest
import torch

import float8_ref as ref
import layer_ref
import paper_2608_16308_amd as dbs
from gpu_helpers import log
from paper_2608_16308_amd import Blocks8, Norm

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    return dbs.LayerContext()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, shape, dt, scale=1.0, pad=0, offset=0):
    rows, cols = shape
    buf = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=dt, device="cuda")
    v = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(shape, generator=g, device="cuda") * scale)
    return v


def same_blocks(c, x, label):
    """c: the blocks of the CPU tensor x."""
    codes, exps = ref.pack(x, c.block)
    got, gexps = ref.held(c)
    assert torch.equal(gexps, exps), f"{label}: exponents"
    ref.same_codes(got, codes, label)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_every_number(ctx, dt):
    """All 65536 bit patterns of the type, beside others of all sizes."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dt).view(256, 256)
    g = torch.Generator().manual_seed(5)
    mixed = x.reshape(-1)[torch.randperm(65536, generator=g)].view(256, 256)
    for v in (x, x.t().contiguous(), mixed):
        for block in ("row", "tile"):
            for across in (False, True):
                c = ctx.pack8(v.cuda(), block=block, across=across)
                same_blocks(c, v.t().contiguous() if across else v, f"{dt} {block} {across}")
                u, w = ctx.unpack8(c).cpu(), ref.unpacked(c)
                nan = w.isnan()
                assert torch.equal(u.isnan(), nan) and torch.equal(u[~nan], w[~nan])


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1), (8, 8)])
@pytest.mark.parametrize("size", [(1, 1), (1, 128), (2, 129), (127, 7), (128, 128), (129, 640), (300, 1000), (5, 4099), (1031, 513)], ids=str)
def test_pack(ctx, size, pad, offset, dt):
    g = gen(size[0] * 3 + size[1])
    x = rnd(g, size, dt, 3.0, pad, offset)
    for block in ("row", "tile"):
        for across in (False, True):
            c = ctx.pack8(x, block=block, across=across)
            v = x.cpu().t().contiguous() if across else x.cpu()
            assert c.shape == tuple(v.shape) and c.dtype == dt
            same_blocks(c, v, f"{size} {block} {across}")
            y = rnd(g, c.shape, dt, 1.0, pad, offset)
            assert torch.equal(ctx.unpack8(c, y=y).cpu(), ref.unpacked(c)) and torch.equal(ctx.unpack8(c), y)


# tokens, n_in, n_out: one of each, blocks' and tiles' edges, few tokens, long sums
SIZES = [(1, 1, 1), (1, 128, 64), (1, 4096, 513), (2, 33, 31), (3, 257, 320), (8, 1024, 1000), (16, 72, 48), (17, 200, 96), (31, 8, 7),
         (64, 128, 256), (65, 4104, 130), (127, 63, 129), (130, 136, 264), (257, 512, 260), (300, 1001, 517), (520, 264, 776),
         (5, 9000, 40), (1030, 640, 530)]


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear(ctx, size, dt):
    t, n, m = size
    g = gen(t * 7 + n * 3 + m)
    log(f"linear8 {size} {dt}")
    x, w = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5)
    w8, x8 = ctx.pack8(w, block="tile"), ctx.pack8(x)
    vx, vw = ref.of(x), ref.of(w, "tile")
    for bias, res in ((None, None), (rnd(g, (1, m), dt)[0], None), (rnd(g, (1, m), dt)[0], rnd(g, (t, m), dt))):
        y = ctx.linear8(x, w8, bias=bias, residual=res)
        layer_ref.check(y.cpu(), *ref.product(vx, vw, dt, bias, res), f"{size}")
        assert torch.equal(ctx.linear8(x8, w8, bias=bias, residual=res), y)
        if res is not None:
            assert torch.equal(ctx.linear8(x, w8, bias=bias, residual=res, y=res), y)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_backward(ctx, size, dt):
    t, n, m = size
    g = gen(t * 3 + n * 5 + m)
    log(f"linear8 backward {size} {dt}")
    x, w, dy = rnd(g, (t, n), dt), rnd(g, (m, n), dt, n ** -0.5), rnd(g, (t, m), dt)
    w8, x8 = ctx.pack8(w, block="tile"), ctx.pack8(x)
    vw, vdy, vdt = ref.of(w, "tile"), ref.of(dy), ref.of(dy.t().contiguous())
    db = dy.cpu().double().sum(0), dy.cpu().double().abs().sum(0)
    for held in (x, x8):
        xv = x.cpu() if held is x else ref.unpacked(x8)
        vxt = ref.of(xv.t().contiguous())
        got = ctx.linear8_backward(dy, held, w8, bias=True)
        layer_ref.check(got[0].cpu(), *ref.product(vdy, vw.T.contiguous(), dt), f"{size} dx")
        layer_ref.check(got[1].cpu(), *ref.product(vdt, vxt, dt), f"{size} dw")
        layer_ref.check(got[2].cpu(), db[0], layer_ref.rounded(db[0], layer_ref.sum_err(t, db[1]), dt), f"{size} db")
    dx, dw, none = ctx.linear8_backward(dy, None, w8, need_dw=False)
    assert dw is None and none is None and torch.equal(dx, got[0])
    dx, dw, _ = ctx.linear8_backward(dy, x8, w8, need_dx=False)
    assert dx is None and torch.equal(dw, got[1])
    assert torch.equal(ctx.linear8_backward(dy, None, w8, bias=True, need_dx=False, need_dw=False)[2], got[2])


def test_scales_far_apart(ctx):
    """Blocks from 2^-120 to 2^120: the matrix cores apply the scales, and no block
    is lost beside another."""
    dt = torch.bfloat16
    g = gen(3)
    n = 1024
    for t in (3, 40, 300):
        x, w = rnd(g, (t, n), dt), rnd(g, (200, n), dt)
        for k in range(n // 128):
            x[:, 128 * k:128 * k + 128] *= 2.0 ** (30 * k - 110)
            w[:, 128 * k:128 * k + 128] *= 2.0 ** (100 - 30 * k)
        x[0] = 0
        w8 = ctx.pack8(w, block="tile")
        layer_ref.check(ctx.linear8(x, w8).cpu(), *ref.product(ref.of(x), ref.of(w, "tile"), dt), f"{t} scales")
        tiny = (x * 0 + 2.0 ** -130)
        layer_ref.check(ctx.linear8(tiny, ctx.pack8(w * 0 + 2.0 ** 100, block="tile")).cpu(),
                        torch.full((t, 200), n * 2.0 ** -30, dtype=torch.float64),
                        torch.full((t, 200), n * 2.0 ** -38, dtype=torch.float64), "smallest exponents")


def test_nan_stays_in_its_row(ctx):
    g = gen(4)
    for t in (4, 150):
        x, w = rnd(g, (t, 300), torch.float16), rnd(g, (140, 300), torch.float16, 0.1)
        clean = ctx.linear8(x, ctx.pack8(w, block="tile"))
        x[1, 7], x[2, 299], w[5, 100] = float("nan"), float("inf"), float("-inf")
        bad = torch.zeros((t, 140), dtype=torch.bool, device="cuda")
        bad[1], bad[2], bad[:, 5] = True, True, True
        y = ctx.linear8(x, ctx.pack8(w, block="tile"))
        assert torch.equal(y.isnan(), bad)
        assert torch.equal(y[~bad], clean[~bad])  # (the other values of the block keep their scale: infinities do not set it)


def test_rows_around_outputs_stay(ctx):
    g = gen(6)
    for t, n, m in ((3, 200, 100), (70, 300, 130), (300, 260, 270)):
        buf = torch.full((t + 2, m + 16), 7.0, dtype=torch.float16, device="cuda")
        out = buf[1:t + 1, 8:8 + m]
        around = torch.ones_like(buf, dtype=torch.bool)
        around[1:t + 1, 8:8 + m] = False
        x, w8 = rnd(g, (t, n), torch.float16), ctx.pack8(rnd(g, (m, n), torch.float16), block="tile")
        y = ctx.linear8(x, w8)
        ctx.linear8(x, w8, y=out)
        assert torch.equal(out, y) and bool((buf[around] == 7.0).all())
        ctx.unpack8(ctx.pack8(y), y=out)
        assert bool((buf[around] == 7.0).all())


def test_nothing(ctx):
    z = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for t, n, m in ((0, 64, 32), (3, 0, 32), (3, 64, 0), (0, 0, 0)):
        w8 = ctx.pack8(z(m, n), block="tile")
        bias = torch.ones(m, dtype=torch.bfloat16, device="cuda")
        for x in (z(t, n), ctx.pack8(z(t, n))):
            y = ctx.linear8(x, w8, bias=bias)
            assert y.shape == (t, m) and (n > 0 or bool((y == 1).all()))
            dx, dw, db = ctx.linear8_backward(z(t, m), x, w8, bias=True)
            assert dx.shape == (t, n) and dw.shape == (m, n) and db.shape == (m,)
            for v in ((dx,) if m == 0 else ()) + ((dw, db) if t == 0 else ()):
                assert float(v.float().abs().sum()) == 0
        assert ctx.unpack8(w8).shape == (m, n) and ctx.pack8(z(t, n), across=True).shape == (n, t)


def test_one_token_and_blocks_by_hand(ctx):
    g = gen(7)
    x, w = rnd(g, (1, 500), torch.float16), rnd(g, (60, 500), torch.float16)
    w8 = ctx.pack8(w, block="tile")
    y = ctx.linear8(x, w8)
    assert torch.equal(ctx.linear8(x[0], w8), y[0])
    codes, exps = ref.pack(w.cpu(), "tile")
    own = Blocks8(codes.cuda().view(torch.float8_e4m3fn), exps.cuda(), "tile", (60, 500), torch.float16)
    assert torch.equal(ctx.linear8(x, own), y) and own.nbytes() == 60 * 512 + 4


@pytest.mark.parametrize("n", [1, 100, 512, 1111, 4096, 5003, 40000])
def test_a_run_of_a_block(ctx, n):
    """norm -> product -> join -> product, with the results in 8 bits passed on: each
    the same as by separate calls, and the whole the formulas'."""
    dt = torch.bfloat16
    g = gen(n)
    t, m = 37, 200
    x, nm = rnd(g, (t, n), dt, 2.0), Norm(rnd(g, (1, n), dt)[0], None, eps=1e-5)
    h8, h = ctx.norm(x, nm, to8=True), ctx.norm(x, nm)
    same_blocks(h8, h.cpu(), "norm to 8 bits")
    w8, d8 = ctx.pack8(rnd(g, (m, n), dt, n ** -0.5), block="tile"), ctx.pack8(rnd(g, (n, m), dt, m ** -0.5), block="tile")
    u = ctx.linear8(h8, w8)
    assert torch.equal(u, ctx.linear8(h, w8))
    layer_ref.check(u.cpu(), *ref.product(ref.of(h), ref.values(w8), dt), "first product")
    branch = ctx.linear8(u, d8)
    args = dict(after=nm, before=nm, gate=nm.weight, p=0.1, rng=(3, 4))
    s, k8 = ctx.join(branch, x, to8=True, **args)
    s2, k = ctx.join(branch, x, **args)
    assert torch.equal(s, s2)
    same_blocks(k8, k.cpu(), "join to 8 bits")
    # back
    dy, ds = rnd(g, (t, m), dt), rnd(g, (t, n), dt)
    dk, dw, _ = ctx.linear8_backward(dy, k8, w8)
    assert torch.equal(dw, ctx.linear8_backward(dy, ctx.unpack8(k8), w8)[1])
    d = ctx.join_backward(ds, dk, branch, s, **args)
    du, dd, _ = ctx.linear8_backward(d.branch, u, d8)
    dh, _, _ = ctx.linear8_backward(du, h8, w8)
    dx, dn, _ = ctx.norm_backward(dh, x, nm, add=d.residual)
    assert all(bool(v.isfinite().all()) for v in (dx, dn, dd, dw, d.gate, d.after_weight, d.before_weight))


def test_captured(ctx):
    side = torch.cuda.Stream()
    own = dbs.LayerContext(side)
    g = gen(13)
    dt = torch.bfloat16
    x, dy = rnd(g, (200, 520), dt), rnd(g, (200, 392), dt)
    w8 = ctx.pack8(rnd(g, (392, 520), dt, 0.05), block="tile")
    step = lambda c: [c.linear8(x, w8), c.linear8(x[:3], w8), *c.linear8_backward(dy, x, w8, bias=True)]  # noqa: E731
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(own)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(own)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        dy.copy_(torch.randn(dy.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step(ctx))), i


def test_no_graph(ctx):
    g = gen(14)
    x, w8 = rnd(g, (20, 64), torch.float16), ctx.pack8(rnd(g, (40, 64), torch.float16), block="tile")
    out = ctx.linear8(x.clone().requires_grad_(), w8)
    with pytest.raises(dbs.DbsError) as e:
        out.float().sum().backward()
    assert "linear8_backward" in str(e.value)


def test_other_stream():
    side = torch.cuda.Stream()
    own, ctx = dbs.LayerContext(side), dbs.LayerContext()
    g = gen(15)
    x, dy = rnd(g, (70, 900), torch.float16), rnd(g, (70, 300), torch.float16)
    w = rnd(g, (300, 900), torch.float16)

    def step(c):
        w8, x8 = c.pack8(w, block="tile"), c.pack8(x)
        return [c.linear8(x8, w8), c.linear8(x, w8), c.linear8(x[:1], w8), *c.linear8_backward(dy, x8, w8, bias=True), c.unpack8(w8)]
    want = step(ctx)
    side.wait_stream(torch.cuda.current_stream())
    got = step(own)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_of_the_other_type(ctx):
    """(a block's values are the same numbers in both)"""
    g = gen(16)
    w8 = ctx.pack8(rnd(g, (136, 260), torch.float16), block="tile")
    other = Blocks8(w8.codes, w8.exponents, "tile", w8.shape, torch.bfloat16)
    for t in (2, 150):
        x, dy = rnd(g, (t, 260), torch.bfloat16), rnd(g, (t, 136), torch.bfloat16)
        assert torch.equal(ctx.linear8(x, w8), ctx.linear8(x, other))
        for a, b in zip(ctx.linear8_backward(dy, x, w8), ctx.linear8_backward(dy, x, other)):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_offsets_past_32_bits(ctx):
    """Rows more than 2^31 elements apart: the same results as of rows beside each other."""
    dt, (n, m) = torch.float16, (1003, 333)
    g = gen(17)
    w8 = ctx.pack8(rnd(g, (m, n), dt, n ** -0.5), block="tile")
    far = (1 << 31) + 24
    buf = torch.empty(2 * far + 8 * n, dtype=dt, device="cuda")
    x, r, y = (buf.as_strided((3, k), (far, 1), i * (n + 1)) for i, k in enumerate((n, m, m)))
    x.copy_(rnd(g, (3, n), dt)), r.copy_(rnd(g, (3, m), dt))
    xc, rc = x.contiguous(), r.contiguous()
    for across in (False, True):
        a, b = ctx.pack8(x, across=across), ctx.pack8(xc, across=across)
        assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.exponents, b.exponents)
    assert torch.equal(ctx.linear8(x, w8, residual=r, y=y), ctx.linear8(xc, w8, residual=rc))
    assert torch.equal(ctx.unpack8(ctx.pack8(rc), y=y), ctx.unpack8(ctx.pack8(rc)))
    for a, b in zip(ctx.linear8_backward(r, x, w8, bias=True), ctx.linear8_backward(rc, xc, w8, bias=True)):
        assert torch.equal(a, b)
    # many tokens, with codes of more than 2^31 bytes of each factor's side
    t, n = 17000, 130000
    x8 = ctx.pack8(torch.zeros((t, n), dtype=dt, device="cuda"))
    last = rnd(g, (300, n), dt)
    part = ctx.pack8(last)
    x8.codes[-300:].view(torch.uint8).copy_(part.codes.view(torch.uint8))
    x8.exponents[-300:].copy_(part.exponents)
    w8 = ctx.pack8(rnd(g, (40, n), dt, n ** -0.5), block="tile")
    y = ctx.linear8(x8, w8)
    want, err = ref.product(ref.values(part), ref.values(w8), dt)
    layer_ref.check(y[-300:].cpu(), want, err, "the last of many tokens")
    assert float(y[:-300].float().abs().max()) == 0.0


def test_captured_in_parts(ctx):
    """A sum that several workgroups share, through the context's workspace, in a graph."""
    side = torch.cuda.Stream()
    own = dbs.LayerContext(side)
    g = gen(18)
    dt = torch.float16
    x, w8 = rnd(g, (40, 9000), dt), ctx.pack8(rnd(g, (264, 9000), dt, 0.01), block="tile")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        own.linear8(x, w8)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = own.linear8(x, w8), own.linear8(x[:33], w8)
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], ctx.linear8(x, w8)) and torch.equal(out[1], ctx.linear8(x[:33], w8)), i
        torch.cuda.synchronize()
