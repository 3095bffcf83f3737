"""Norms, joins, dropout and their gradients on the GPU against their definitions in 64 bits."""
import pytest
import torch

import edges_ref as ref
import layer_ref
import paper_2608_16308_amd as dbs
from gpu_helpers import log
from paper_2608_16308_amd import Norm

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
# one of each, around the chunks of 8, the lanes' and the waves' edges, rows of
# several workgroups' lengths, many rows
SIZES = [(1, 1), (1, 7), (2, 8), (3, 9), (1, 4096), (3, 257), (5, 512), (4, 513), (4, 1000), (7, 1111), (64, 128), (33, 4096), (130, 2048),
         (2, 5003), (3, 8200), (2, 14336), (1, 16385), (2, 32769), (2, 70001), (300, 64), (1025, 24), (700, 520)]


@pytest.fixture(scope="module")
def ctx():
    return dbs.LayerContext()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, shape, dt, scale=1.0, mean=0.0, pad=0, offset=0):
    """N(mean, scale) in a buffer with rows `pad` longer that starts `offset` elements
    into it; what lies around is NaN."""
    rows, cols = shape
    buf = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=dt, device="cuda")
    v = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(shape, generator=g, device="cuda") * scale + mean)
    return v


def make_norm(g, n, dt, kind, weight=True, bias=True, offset=0):
    return Norm(rnd(g, (1, n), dt, 0.2, 1.0, offset=offset)[0] if weight else None,
                rnd(g, (1, n), dt, 0.2, offset=offset)[0] if bias else None, kind=kind, eps=1e-5)


def check(got, want, label):
    layer_ref.check(got.cpu(), *want, label)


def check_all(got, want, label):
    for name, v in want.items():
        check(getattr(got, name), v, f"{label} {name}")
    for name in got._fields:
        assert name in want or getattr(got, name) is None, name


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_norm(ctx, size, dt):
    g = gen(size[0] * 7 + size[1])
    log(f"norm {size} {dt}")
    for kind in ("rms", "layer"):
        for weight, bias in ((True, True), (True, False), (False, False), (False, True)):
            nm = make_norm(g, size[1], dt, kind, weight, bias)
            x, dy, add = rnd(g, size, dt, 2.0, 0.5), rnd(g, size, dt), rnd(g, size, dt)
            label = f"{size} {kind} {weight} {bias}"
            check(ctx.norm(x, nm), ref.norm(x, nm), label)
            for more in (None, add):
                want = ref.norm_backward(dy, x, nm, more)
                dx, dw, db = ctx.norm_backward(dy, x, nm, add=more)
                got = {k: v for k, v in (("dx", dx), ("dweight", dw), ("dbias", db)) if v is not None}
                assert got.keys() == want.keys()
                for k, v in got.items():
                    check(v, want[k], f"{label} {k}")
    dx, dw, db = ctx.norm_backward(dy, x, nm, need_dw=False)
    assert dw is None and db is None and torch.equal(dx, ctx.norm_backward(dy, x, nm)[0])
    assert ctx.norm_backward(dy, x, nm, need_dx=False)[0] is None


FORMS = [dict(after="rms", before="rms", gate="vector", scale=0.75, p=0.1), dict(after="layer", before="layer", gate="token", scale=1.0, p=0.5),
         dict(after=None, before="rms", gate=None, scale=1.0, p=0.0), dict(after="layer", before=None, gate=None, scale=-2.0, p=0.25),
         dict(after=None, before=None, gate="token", scale=0.0, p=0.3), dict(after=None, before="layer", gate="vector", scale=1.0, p=1.0)]


def make_join(g, size, dt, form, **at):
    t, n = size
    norm = lambda k: None if k is None else make_norm(g, n, dt, k, offset=at.get("offset", 0))  # noqa: E731
    gate = {None: lambda: None, "vector": lambda: rnd(g, (1, n), dt, 0.3, 0.5, offset=at.get("offset", 0))[0],
            "token": lambda: rnd(g, size, dt, 0.3, 0.5, **at)}[form["gate"]]()
    return dict(after=norm(form["after"]), before=norm(form["before"]), gate=gate, scale=form["scale"], p=form["p"],
                rng=(t + (n << 35), 9 + (t << 34)))


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_join(ctx, size, dt):
    g = gen(size[0] * 5 + size[1])
    log(f"join {size} {dt}")
    for form in FORMS:
        args = make_join(g, size, dt, form)
        branch, residual = rnd(g, size, dt, 2.0, 0.5), rnd(g, size, dt, 3.0)
        want = ref.join(branch, residual, **args)
        stream, h = ctx.join(branch, residual, **args)
        check(stream, want["stream"], f"{size} {form} stream")
        assert (h is None) == (args["before"] is None)
        if h is not None:
            check(h, want["h"], f"{size} {form} h")
        ds, dh = rnd(g, size, dt), None if h is None else rnd(g, size, dt)
        check_all(ctx.join_backward(ds, dh, branch, stream, **args), ref.join_backward(ds, dh, branch, stream, **args), f"{size} {form}")
    few = ctx.join_backward(ds, dh, branch, stream, need_dw=False, **args)
    full = ctx.join_backward(ds, dh, branch, stream, **args)
    assert few.gate is None and few.before_weight is None
    assert torch.equal(few.residual, full.residual) and torch.equal(few.branch, full.branch)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_join_backward_without_a_stream_gradient(ctx, dt):
    size = (9, 700)
    g = gen(4)
    args = make_join(g, size, dt, FORMS[0])
    branch, stream, dh = rnd(g, size, dt), rnd(g, size, dt), rnd(g, size, dt)
    check_all(ctx.join_backward(None, dh, branch, stream, **args), ref.join_backward(None, dh, branch, stream, **args), "no dstream")
    # neither gate nor norms: branch and stream are not read
    ds = rnd(g, size, dt)
    plain = dict(after=None, before=None, gate=None, scale=0.5, p=0.2, rng=(1, 2))
    check_all(ctx.join_backward(ds, None, None, None, **plain), ref.join_backward(ds, None, None, None, **plain), "plain")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_dropout(ctx, size, dt):
    g = gen(size[0] + size[1])
    x = rnd(g, size, dt, 2.0)
    for p, rng in ((0.1, (0, 0)), (0.5, (3 << 50, 1 << 40)), (0.0, None), (1.0, (5, 6)), (1e-6, (1, 1)), (0.99999, (2 ** 64 - 1, 2 ** 64 - 1))):
        f = ref.factor(*size, p, rng or (0, 0))
        want = x.cpu().double() * f
        # fp16: 65504 and half a step up, 65520 and more, round to infinity (x 65536 where p is nearly 1)
        want = torch.where(want.abs() >= 65520, torch.sign(want) * float("inf"), want) if dt == torch.float16 else want
        got = ctx.dropout(x, p, rng)
        # (one product in 32 bits by a factor that is itself rounded to 32)
        check(got, (want, layer_ref.rounded(want, 2.0 ** -23 * want.abs(), dt)), f"{size} {p}")
        assert torch.equal((got == 0).cpu(), (want == 0))


# rows in wider buffers, bases off their alignment
@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 0), (8, 0), (64, 8), (5, 3), (8, 4)])
@pytest.mark.parametrize("size", [(1, 256), (6, 1000), (37, 512), (20, 4099), (3, 33000)], ids=str)
def test_strides_and_alignment(ctx, size, pad, offset, dt):
    g = gen(size[0] + size[1] + 17 * pad + offset)
    log(f"edges strides {size} pad {pad} offset {offset} {dt}")
    at = dict(pad=pad, offset=offset)
    make = lambda *a: rnd(g, size, dt, *a, **at)  # noqa: E731
    nm = make_norm(g, size[1], dt, "layer", offset=offset)
    x, dy, add = make(2.0), make(), make()
    y = make()
    want = ref.norm(x, nm)
    check(ctx.norm(x, nm, y=y), want, "norm into y")
    z = x.clone()
    check(ctx.norm(z, nm, y=z), want, "norm in place")
    for k, v in zip(("dx", "dweight", "dbias"), ctx.norm_backward(dy, x, nm, add=add)):
        check(v, ref.norm_backward(dy, x, nm, add)[k], k)
    for form in FORMS[:2]:
        args = make_join(g, size, dt, form, **at)
        branch, residual = make(2.0), make(3.0)
        want = ref.join(branch, residual, **args)
        out = make()
        stream, h = ctx.join(branch, residual, stream=out, **args)
        assert stream.data_ptr() == out.data_ptr()
        check(stream, want["stream"], "join into stream")
        check(h, want["h"], "join h")
        inplace = torch.nn.functional.pad(residual, (0, pad))[:, :size[1]] if pad else residual.clone()
        s2, h2 = ctx.join(branch, inplace, stream=inplace, **args)
        assert torch.equal(s2, stream) and torch.equal(h2, h)
        ds, dh = make(), make()
        check_all(ctx.join_backward(ds, dh, branch, stream, **args), ref.join_backward(ds, dh, branch, stream, **args), "join backward")
    f = ref.factor(*size, 0.3, (1, 2))
    want = x.cpu().double() * f
    bound = layer_ref.rounded(want, 2.0 ** -23 * want.abs(), dt)
    check(ctx.dropout(x, 0.3, (1, 2), y=y), (want, bound), "dropout into y")
    check(ctx.dropout(z.copy_(x), 0.3, (1, 2), y=z), (want, bound), "dropout in place")


def test_rows_around_outputs_stay(ctx):
    """What lies beside and behind an output is left as it was."""
    g = gen(15)
    for t, n in ((3, 100), (2, 33001), (5, 4096), (4, 5003)):
        buf = torch.full((t + 2, n + 16), 30000.0, dtype=torch.float16, device="cuda")
        x = rnd(g, (t, n), torch.float16)
        out = buf[1:t + 1, 8:8 + n]
        around = torch.ones_like(buf, dtype=torch.bool)
        around[1:t + 1, 8:8 + n] = False
        for call in (lambda: ctx.norm(x, Norm(), y=out), lambda: ctx.dropout(x, 0.5, (1, 2), y=out),
                     lambda: ctx.join(x, x.clone(), before=Norm(), stream=out)):
            call()
            assert bool((buf[around] == 30000.0).all()) and not bool((out == 30000.0).any())


@pytest.mark.parametrize("n", [300, 4096, 33000])
def test_values_at_the_ends(ctx, n):
    """Large means, squares beyond 32 bits, zeros, infinities and NaN: a row touches no other."""
    g = gen(n)
    for kind in ("rms", "layer"):
        nm = Norm(None, None, kind=kind, eps=1e-5)
        x = torch.randn((9, n), generator=g, device="cuda")
        x[0] = 0
        x[1] = 1000 + x[1]
        x[2] *= 1e30
        x[3] = 1e37 * torch.sign(x[3])
        x[4, n // 2] = float("inf")
        x[5, 0] = float("nan")
        x[6] *= 1e-30
        x[7] = 3.0
        x = x.bfloat16()
        got = ctx.norm(x, nm)
        keep = [0, 1, 2, 3, 6, 7, 8]
        check(got[keep], ref.norm(x[keep], nm), f"{kind} finite rows")
        assert bool(got[5].isnan().all())
        # x / inf: zeros, and NaN where inf / inf (the layer's mean is infinite too)
        assert bool(got[4].isnan().all()) if kind == "layer" else bool(got[4, n // 2].isnan()) and int((got[4] != 0).sum()) == 1
        dy = torch.randn((9, n), generator=g, device="cuda").bfloat16()
        keep = [0, 1, 2, 3, 6, 8]
        dx, _, _ = ctx.norm_backward(dy, x, nm)
        check(dx[keep], ref.norm_backward(dy[keep], x[keep], nm)["dx"], f"{kind} gradients of finite rows")
        assert bool(dx[5].isnan().all())
    # what is dropped is zero, whatever it was
    x = torch.full((4, n), float("nan"), dtype=torch.float16, device="cuda")
    y = ctx.dropout(x, 0.5, (1, 2)).cpu()
    assert torch.equal(y == 0, ref.factor(4, n, 0.5, (1, 2)) == 0)
    s, _ = ctx.join(x, torch.ones_like(x), p=0.5, rng=(1, 2))
    assert torch.equal(s.cpu() == 1, ref.factor(4, n, 0.5, (1, 2)) == 0)


def test_no_rows_and_no_columns(ctx):
    for t, n in ((0, 64), (3, 0), (0, 0)):
        x = torch.empty((t, n), dtype=torch.float16, device="cuda")
        nm = Norm(torch.ones(n, dtype=torch.float16, device="cuda"), torch.ones(n, dtype=torch.float16, device="cuda"), kind="layer")
        assert ctx.norm(x, nm).shape == (t, n)
        assert ctx.norm(x, nm, to8=True).shape == (t, n)
        dx, dw, db = ctx.norm_backward(x, x, nm)
        assert dx.shape == (t, n) and float(dw.abs().sum() + db.abs().sum()) == 0
        s, h = ctx.join(x, x.clone(), after=nm, before=nm, gate=nm.weight, p=0.1, rng=(1, 2))
        assert s.shape == h.shape == (t, n)
        d = ctx.join_backward(x, x, x, x, after=nm, before=nm, gate=nm.weight, p=0.1, rng=(1, 2))
        for v in (d.gate, d.after_weight, d.before_bias):
            assert v.shape == (n,) and float(v.abs().sum()) == 0
        assert ctx.dropout(x, 0.1, (1, 2)).shape == (t, n)


def test_one_token(ctx):
    g = gen(8)
    x, r = (rnd(g, (1, 1000), torch.float16)[0] for _ in range(2))
    nm = make_norm(g, 1000, torch.float16, "rms")
    assert torch.equal(ctx.norm(x, nm), ctx.norm(x[None], nm)[0])
    s, h = ctx.join(x, r, before=nm, gate=nm.weight)
    s2, h2 = ctx.join(x[None], r[None], before=nm, gate=nm.weight)
    assert s.shape == h.shape == (1000,) and torch.equal(s, s2[0]) and torch.equal(h, h2[0])
    assert torch.equal(ctx.dropout(x, 0.5, (1, 2)), ctx.dropout(x[None], 0.5, (1, 2))[0])


def test_same_call_same_bits(ctx):
    g = gen(9)
    size, dt = (777, 1111), torch.bfloat16
    args = make_join(g, size, dt, FORMS[0])
    branch, residual, ds, dh = (rnd(g, size, dt) for _ in range(4))
    first = None
    for _ in range(3):
        s, h = ctx.join(branch, residual, **args)
        out = [s, h, *ctx.join_backward(ds, dh, branch, s, **args)]
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_captured(ctx):
    """A join and its gradients in a graph, replayed with other inputs and another
    seed in device memory, eager work of the program between the replays."""
    side = torch.cuda.Stream()
    own = dbs.LayerContext(side)
    g = gen(10)
    size, dt = (65, 2056), torch.bfloat16
    args = make_join(g, size, dt, FORMS[0])
    rng = torch.tensor([5, 6], dtype=torch.int64, device="cuda")
    args["rng"] = rng
    x = [rnd(g, size, dt) for _ in range(4)]

    def step(c):
        s, h = c.join(x[0], x[1], **args)
        d = c.join_backward(x[2], x[3], x[0], s, **args)
        n = c.norm_backward(x[3], x[1], args["before"], add=x[2])
        return [s, h, c.dropout(h, 0.2, rng), *d, *n]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(own)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(own)
    for i in range(4):
        for v in x:
            v.copy_(torch.randn(size, generator=g, device="cuda"))
        rng.copy_(torch.tensor([i * 11, i + (1 << 40)], device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step(ctx)
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b)), i
    args["rng"] = (33, 3 + (1 << 40))
    s, _ = ctx.join(x[0], x[1], **args)
    assert torch.equal(s, out[0])


def test_other_stream():
    side = torch.cuda.Stream()
    own = dbs.LayerContext(side)
    g = gen(11)
    x, nm = rnd(g, (50, 3000), torch.float16), make_norm(g, 3000, torch.float16, "layer")
    want = dbs.LayerContext().norm(x, nm)
    side.wait_stream(torch.cuda.current_stream())
    y = own.norm(x, nm)
    d = own.join_backward(x, x, x, x, after=nm, before=nm, gate=nm.weight)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    ref_d = dbs.LayerContext().join_backward(x, x, x, x, after=nm, before=nm, gate=nm.weight)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(d, ref_d))


def test_no_graph(ctx):
    g = gen(12)
    x, nm = rnd(g, (4, 64), torch.float16), make_norm(g, 64, torch.float16, "rms")
    p = Norm(nm.weight.clone().requires_grad_(), nm.bias)
    for out, word in ((ctx.norm(x, p), "norm_backward"), (ctx.join(x, x.clone(), before=p)[1], "join_backward"),
                      (ctx.dropout(x.clone().requires_grad_(), 0.5, (1, 2)), "same call")):
        assert out.requires_grad
        with pytest.raises(dbs.DbsError) as e:
            out.float().sum().backward()
        assert word in str(e.value)
    assert not ctx.norm(x, nm).requires_grad


def test_offsets_past_32_bits(ctx):
    """Rows more than 2^31 elements apart: the same results as of rows beside each other."""
    dt, (t, n) = torch.float16, (3, 1003)
    g = gen(15)
    far = (1 << 31) + 8
    buf = torch.empty(2 * far + 8 * n, dtype=dt, device="cuda")
    spread = [buf.as_strided((t, n), (far, 1), i * (n + 1)) for i in range(7)]
    x = [rnd(g, (t, n), dt) for _ in range(5)]
    for a, b in zip(spread, x):
        a.copy_(b)
    args = dict(after=make_norm(g, n, dt, "layer"), before=make_norm(g, n, dt, "rms"), p=0.2, rng=(7, 8))
    s, h = ctx.join(x[0], x[1], gate=x[2], **args)
    s2, h2 = ctx.join(spread[0], spread[1], gate=spread[2], stream=spread[5], **args)
    assert torch.equal(s2, s) and torch.equal(h2, h)
    d = ctx.join_backward(x[3], x[4], x[0], s, gate=x[2], **args)
    d2 = ctx.join_backward(spread[3], spread[4], spread[0], s2, gate=spread[2], **args)
    assert all(torch.equal(a, b) for a, b in zip(d, d2))
    nm = args["before"]
    assert torch.equal(ctx.norm(spread[0], nm, y=spread[6]), ctx.norm(x[0], nm))
    assert torch.equal(ctx.dropout(spread[0], 0.3, (1, 2), y=spread[6]), ctx.dropout(x[0], 0.3, (1, 2)))
    for a, b in zip(ctx.norm_backward(spread[3], spread[0], nm, add=spread[4]), ctx.norm_backward(x[3], x[0], nm, add=x[4])):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    long = 20000  # (and the rows that registers do not hold)
    a = buf.as_strided((t, long), (far - long, 1), 0)
    a.copy_(torch.randn((t, long), generator=g, device="cuda"))
    nm = make_norm(g, long, dt, "layer")
    b = a.contiguous()
    assert torch.equal(ctx.norm(a, nm), ctx.norm(b, nm))
    for u, v in zip(ctx.norm_backward(a, a, nm), ctx.norm_backward(b, b, nm)):
        assert torch.equal(u, v)


def test_more_than_32_bits_of_elements(ctx):
    """The last rows of a matrix of more than 2^31 elements, where they are and alone."""
    t, n = 70001, 31000
    x = torch.zeros((t, n), dtype=torch.bfloat16, device="cuda")
    last = x[-3:]
    last.copy_(torch.randn((3, n), generator=gen(16), device="cuda"))
    nm = Norm(None, None, kind="layer", eps=1e-5)
    assert torch.equal(ctx.norm(x, nm)[-3:], ctx.norm(last, nm))
    y = ctx.dropout(x, 0.25, (5, 6))[-3:]
    want = last.cpu().double() * ref.factor(3, n, 0.25, (5, 6), first=t - 3)
    check(y, (want, layer_ref.rounded(want, 2.0 ** -23 * want.abs(), torch.bfloat16)), "dropout")


# several rows one after the other for each team of waves, of each number of them
@pytest.mark.parametrize("size", [(3001, 40), (1600, 905), (1100, 1501), (1100, 2048), (560, 2304), (530, 4090), (525, 5003), (300, 6151), (290, 8192),
                                  (270, 9001), (270, 15000)], ids=str)
def test_many_rows(ctx, size):
    g = gen(size[1])
    log(f"many rows {size}")
    for dt, form in ((torch.bfloat16, FORMS[0]), (torch.float16, FORMS[1]), (torch.float16, FORMS[3]), (torch.bfloat16, FORMS[5])):
        args = make_join(g, size, dt, form)
        branch, residual, ds = rnd(g, size, dt, 2.0, 0.5), rnd(g, size, dt, 3.0), rnd(g, size, dt)
        want = ref.join(branch, residual, **args)
        stream, h = ctx.join(branch, residual, **args)
        check(stream, want["stream"], f"{size} {form} stream")
        dh = None
        if h is not None:
            check(h, want["h"], f"{size} {form} h")
            dh = rnd(g, size, dt)
        check_all(ctx.join_backward(ds, dh, branch, stream, **args), ref.join_backward(ds, dh, branch, stream, **args), f"{size} {form}")
    for kind in ("rms", "layer"):
        nm = make_norm(g, size[1], dt, kind)
        check(ctx.norm(branch, nm), ref.norm(branch, nm), f"{size} {kind}")
        for k, v in zip(("dx", "dweight", "dbias"), ctx.norm_backward(ds, branch, nm, add=residual)):
            check(v, ref.norm_backward(ds, branch, nm, residual)[k], f"{size} {kind} {k}")


@pytest.mark.parametrize("n", [200, 1111, 4096, 9000, 20000])
def test_means_far_from_zero(ctx, n):
    """Rows far from zero, and ones whose parts lie far apart."""
    g = gen(17 + n)
    size, dt = (5, n), torch.float16
    far = rnd(g, size, dt, 1.0, 900.0)
    parts = rnd(g, size, dt, 1.0) + (torch.arange(n, device="cuda") // 512 % 3 - 1) * 1000.0
    for x in (far, parts.to(dt)):
        nm, dy = make_norm(g, n, dt, "layer"), rnd(g, size, dt)
        check(ctx.norm(x, nm), ref.norm(x, nm), f"{n}")
        for k, v in zip(("dx", "dweight", "dbias"), ctx.norm_backward(dy, x, nm)):
            check(v, ref.norm_backward(dy, x, nm)[k], f"{n} {k}")
        args = dict(after=nm, before=nm, gate=None, scale=1.0, p=0.0, rng=None)
        check_all(ctx.join_backward(dy, dy, x, x, **args), ref.join_backward(dy, dy, x, x, **args), f"{n} join")
