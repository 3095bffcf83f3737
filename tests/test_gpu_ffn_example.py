"""The feed-forward block of examples/ runs: training lowers the loss, and
serving the pruned block agrees with the dense layers."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("sizes", [(256, 704, 384), (130, 333, 200)])
def test_ffn_block(sizes):
    import ffn_block
    width, hidden, tokens = sizes
    losses, off = ffn_block.main(["--width", str(width), "--hidden", str(hidden), "--tokens", str(tokens), "--steps", "12"])
    assert losses[-1] < 0.8 * losses[0], losses
    # two float16 results: each rounded once after h (a unit in the last place is 2^-10), and y after the residual
    assert off < 2e-3
