"""Norms of rows so small that their squares leave the range of 32 bits, with an eps that
does not hide it, on the GPU against 64 bits."""
import pytest
import torch

import edges_ref as ref
import layer_ref
from gpu_helpers import log
from paper_2608_16308_amd import Norm
from test_gpu_edges import ctx, gen, rnd  # noqa: F401

pytestmark = pytest.mark.gpu
# sizes of a row's numbers; 2^-131: all of them below bf16's normal range, some are zeros
SCALES = [2.0 ** -50, 2.0 ** -61, 2.0 ** -66, 2.0 ** -75, 2.0 ** -100, 2.0 ** -120, 2.0 ** -131]
# chunks of a lane that are read and worked on differently, teams of one wave and more, rows that registers do not hold
COLUMNS = [7, 8, 300, 1111, 4096, 7001, 9000, 20001]


class Row(ref.Row):
    """Gradients g that are themselves below 2^-126 are held in steps of 2^-149, which the
    division by a tiny row makes large.  In such steps: g = dy w is off by 1/2, the mean of g xh
    by 1 (half a step for a term's part of it, half for the mean), that times xh by |xh| + 1/2, the mean
    of g by 1, each of the two differences by 1/2: together less than 4 + 2 max |xh|."""

    def back(self, dy, edy):
        (dx, edx), dw, db = super().back(dy, edy)
        return (dx, edx + (4 + 2 * self.xh.abs().amax(1, keepdim=True)) * 2.0 ** -149 * self.rstd), dw, db


@pytest.fixture(autouse=True)
def rows(monkeypatch):
    monkeypatch.setattr(ref, "Row", Row)


def check(got, want, label):
    """Values beyond bf16's largest (and half a step) are infinite, those whose bound reaches
    across either."""
    v, e = (t.clone() for t in want)
    got, most = got.cpu().double(), layer_ref.MAX[torch.bfloat16] * (1 + 2.0 ** -9)
    far = v.abs() - e >= most
    v[far] = torch.sign(v[far]) * float("inf")
    near = ~far & (v.abs() + e >= most) & (got == torch.sign(v) * float("inf"))
    v[near] = got[near]
    layer_ref.check(got, v, e, label)


def check_all(got, want, label):
    for name, v in want.items():
        check(getattr(got, name), v, f"{label} {name}")


def make(n, kind, eps):
    """Rows of all scales between ordinary ones, gradients that stay in range."""
    g = gen(n)
    x, dy = rnd(g, (2 * len(SCALES), n), torch.bfloat16), rnd(g, (2 * len(SCALES), n), torch.bfloat16)
    for i, s in enumerate(SCALES):
        x[2 * i] *= s
        dy[2 * i] *= 2.0 ** -12 if s < 2.0 ** -110 else 1.0
    weight = rnd(g, (1, n), torch.bfloat16, 0.2, 1.0)[0]
    return g, x, dy, Norm(weight, None if kind == "rms" else weight.clone(), kind=kind, eps=eps)


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -140, 2.0 ** -124, 2.0 ** -118])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("n", COLUMNS)
def test_norm(ctx, n, kind, eps):  # noqa: F811
    log(f"tiny rows {n} {kind} {eps}")
    _, x, dy, nm = make(n, kind, eps)
    check(ctx.norm(x, nm), ref.norm(x, nm), f"{n} {kind} {eps}")
    want = ref.norm_backward(dy, x, nm)
    for k, v in zip(("dx", "dweight", "dbias"), ctx.norm_backward(dy, x, nm)):
        assert (v is None) == (k not in want)
        if v is not None:
            check(v, want[k], f"{n} {kind} {eps} {k}")


@pytest.mark.parametrize("kinds", [("rms", "rms"), ("layer", "layer"), ("rms", "layer"), ("layer", "rms"), ("rms", None), (None, "rms"), ("layer", None)],
                         ids=str)
@pytest.mark.parametrize("n", COLUMNS)
def test_join(ctx, n, kinds):  # noqa: F811
    """Tiny rows of the branch beside ordinary ones of the stream and the reverse, and both."""
    log(f"tiny rows in a join {n} {kinds}")
    g, branch, ds, after = make(n, kinds[0] or "rms", 0.0)
    _, stream, dh, before = make(n, kinds[1] or "rms", 0.0)
    after, before = after if kinds[0] else None, before if kinds[1] else None
    for roll in (0, 1):
        b, s = branch, stream.roll(roll, 0)
        # (two tiny rows one behind the other would leave the range: the gradient between them is small too)
        d, h = ds, dh.roll(roll, 0)
        args = dict(after=after, before=before, gate=None, scale=1.0, p=0.25, rng=(3, 4))
        if kinds[0] and kinds[1] and roll == 0:
            d = d * 2.0 ** -60
            h = (h.float() * torch.where(s.float().abs().amax(1, True) < 2.0 ** -40, s.float().abs().amax(1, True), 1.0)).bfloat16()
        if before is None:
            h = None
        check_all(ctx.join_backward(d, h, b, s, **args), ref.join_backward(d, h, b, s, **args), f"{n} {kinds} {roll}")
        out, y = ctx.join(b, s * 0, **args)
        want = ref.join(b, s * 0, **args)
        check(out, want["stream"], f"{n} {kinds} stream")
        if before is not None and after is not None:
            check(y, want["h"], f"{n} {kinds} h")


def test_join_of_tiny_streams(ctx):  # noqa: F811
    """A stream that is tiny as a whole, into 16 and into 8 bits."""
    for n in COLUMNS:
        _, x, _, nm = make(n, "rms", 0.0)
        z = torch.zeros_like(x)
        want = ref.join(z, x, None, nm, None, 1.0, 0.0, None)
        s, h = ctx.join(z, x, before=nm)
        check(s, want["stream"], f"{n} stream")
        check(h, want["h"], f"{n} h")
        h8 = ctx.unpack8(ctx.norm(x, nm, to8=True))
        assert torch.equal(h8, ctx.unpack8(ctx.pack8(ctx.norm(x, nm))))


def test_rows_without_spread(ctx):  # noqa: F811
    """Rows of one number: zeros of 0 / sqrt(eps), and NaN of 0 / 0 where eps is 0."""
    for n in COLUMNS:
        x = torch.tensor([0.0, 1.0, 2.0 ** 30, 2.0 ** 100, 2.0 ** -130]).cuda().bfloat16()[:, None].expand(5, n).contiguous()
        for eps in (2.0 ** -140, 2.0 ** -124):
            y = ctx.norm(x, Norm(None, None, kind="layer", eps=eps))
            # (where n is no power of two a mean of n numbers is rounded, and the layer norm shows that)
            if n & (n - 1) == 0:
                assert bool((y == 0).all())
            assert bool((y[0] == 0).all()) and bool((ctx.norm(x, Norm(eps=eps))[0] == 0).all())
        assert bool(ctx.norm(x, Norm(eps=0.0))[0].isnan().all())
