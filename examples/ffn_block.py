"""A feed-forward block trained dense and served pruned.

    h = relu(x Wg^T) * (x Wu^T);  y = h Wd^T + x

1. A few steps of training against the outputs of a fixed teacher: the gated
   layer keeps its projections and its input in 8 bits, and its backward pass
   reads them; the down projection adds the residual in its epilogue.
2. The down weights are pruned to half by magnitude and converted on the GPU.
3. Serving, a token at a time: the gated layer gives an activation most of
   whose entries are zero, and the sparse decode multiplies the others only.

    python examples/ffn_block.py [--width 512] [--hidden 1376] [--tokens 1024] [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_16308_amd as dbs  # noqa: E402


def train(ctx, width, hidden, tokens, steps, rate=0.03):
    """(w_gate, w_up, w_down, losses): float16 layers, 32-bit weights behind them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    layer = lambda m, n: torch.randn((m, n), generator=g, device="cuda") * n ** -0.5  # noqa: E731
    teacher = [w.half() for w in (layer(hidden, width), layer(hidden, width), layer(width, hidden))]
    weights = [w.float() + 0.3 * layer(*w.shape) for w in teacher]
    losses = []
    for _ in range(steps):
        x = torch.randn((tokens, width), generator=g, device="cuda").half()
        target = ctx.linear(ctx.gated(x, teacher[0], teacher[1], act="relu"), teacher[2], residual=x)
        w_gate, w_up, w_down = (w.half() for w in weights)
        h, gate, up = ctx.gated(x, w_gate, w_up, act="relu", save="8bit")
        held = ctx.pack(x)
        y = ctx.linear(h, w_down, residual=x)
        off = y.float() - target.float()
        losses.append(float(off.square().mean()))
        dy = (off / off.numel() ** 0.5).half()
        dh, dw_down, _ = ctx.linear_backward(dy, h, w_down)
        _, dw_gate, dw_up = ctx.gated_backward(dh, held, w_gate, w_up, gate, up, act="relu", need_dx=False)
        for w, d in zip(weights, (dw_gate, dw_up, dw_down)):  # steps of a fixed share of the weights' norm
            w -= rate * w.norm() * d.float() / d.float().norm()
    return [w.half() for w in weights] + [losses]


def prune(w, keep=0.5):
    """w with all but its largest magnitudes of each row set to zero."""
    least = w.abs().float().kthvalue(int(w.shape[1] * (1 - keep)), dim=1).values
    return torch.where(w.abs().float() > least[:, None], w, torch.zeros_like(w))


def serve(ctx, w_gate, w_up, w_down, tokens):
    """Each token through the gated layer and the pruned down projection."""
    down = dbs.Matrix.from_dense(w_down)
    sparse = dbs.Context(down)
    out, active = [], 0.0
    for x in tokens:
        h = ctx.gated(x, w_gate, w_up, act="relu")
        out.append(sparse.spmspv_dense(down, h) + x)
        active += float((h != 0).float().mean()) / len(tokens)
    return torch.stack(out), active


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--width", type=int, default=512)
    p.add_argument("--hidden", type=int, default=1376)
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args(argv)
    ctx = dbs.LayerContext()
    w_gate, w_up, w_down, losses = train(ctx, a.width, a.hidden, a.tokens, a.steps)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    pruned = prune(w_down)
    x = torch.randn((8, a.width), device="cuda").half()
    y, active = serve(ctx, w_gate, w_up, pruned, x)
    dense = ctx.linear(ctx.gated(x, w_gate, w_up, act="relu"), pruned, residual=x)
    off = float((y.float() - dense.float()).norm() / dense.float().norm())
    print(f"served {len(x)} tokens: {100 * active:.0f}% of the activation active, {off:.1e} from the dense layers")
    return losses, off


if __name__ == "__main__":
    main()
