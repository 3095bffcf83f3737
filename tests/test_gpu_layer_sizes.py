"""Layers so wide that their workgroups take more than one launch."""
import pytest
import torch

import paper_2608_16308_amd as dbs
from gpu_helpers import log

pytestmark = pytest.mark.gpu
F16 = torch.float16


def small(n, seed):
    """n whole numbers from -3 to 3, of which sums and products are exact."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(-3, 4, (n,), generator=g, device="cuda", dtype=torch.int8).to(F16)


@pytest.mark.parametrize("t", [1, 2])
def test_forward(t):
    """The kernels for few tokens, eight products a row (2 tokens: a wave to a
    workgroup, whose groups pass 2^32 threads at 2^29 rows)."""
    ctx = dbs.LayerContext()
    n = (1 << 26) + 9 if t == 1 else (1 << 29) + 9
    x = small(t * 8, 1).view(t, 8)
    w = small(n * 8, 2).view(n, 8)
    log(f"gated {t} x 8 -> {n}")
    h = ctx.gated(x, w, w, act="relu")
    step = 1 << 24
    for a in range(0, n, step):
        for r in range(t):
            z = (w[a:a + step].float() * x[r].float()).sum(1)
            assert torch.equal(h[r, a:a + step], (z.clamp(min=0) * z).half()), (r, a)
    if t == 1:
        del h
        m = 2 * n
        log(f"linear 1 x 4 rows of {m}")
        w = torch.cat([w, w])
        y = ctx.linear(x, w)
        for a in range(0, m, step):
            assert torch.equal(y[0, a:a + step].float(), (w[a:a + step].float() * x[0].float()).sum(1)), a


def test_sums_of_the_columns():
    ctx = dbs.LayerContext()
    n = (1 << 28) + 77
    dy, w = small(2 * n, 3).view(2, n), torch.empty((n, 0), dtype=F16, device="cuda")
    log(f"db of {n}")
    _, _, db = ctx.linear_backward(dy, None, w, bias=True, need_dx=False, need_dw=False)
    assert torch.equal(db, dy[0] + dy[1])


def test_weight_gradients():
    """Tiles of the product: 2^23 of each of two matrices, 256 threads a tile."""
    ctx = dbs.LayerContext()
    n = 1 << 30
    x = torch.full((1, 1), 2.0, dtype=F16, device="cuda")
    dh, gate, up = (small(n, s).view(1, n) for s in (4, 5, 6))
    w = up.view(n, 1)  # (not read without dx)
    log(f"dw of {n}")
    _, dwg, dwu = ctx.gated_backward(dh, x, w, w, gate, up, act="none", need_dx=False)
    assert torch.equal(dwg.view(-1), (dh * up * 2).view(-1)) and torch.equal(dwu.view(-1), (dh * gate * 2).view(-1))
