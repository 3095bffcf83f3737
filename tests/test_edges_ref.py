"""The generator's published vectors, and the gradients of the reference against differences (CPU only)."""
import numpy as np
import pytest
import torch

import edges_ref as ref
from paper_2608_16308_amd import Norm


def test_generator():
    """Known answers of Philox4x32-10 (Salmon et al., the authors' test vectors)."""
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((ref.MASK,) * 4, (ref.MASK,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(ref.philox(counter, key)) == want


def test_factor_is_the_generator():
    seed, offset = (7 << 40) + 3, (5 << 33) + 1
    f = ref.factor(5, 21, 0.3, (seed, offset))
    for row in range(5):
        for col in range(21):
            w = ref.philox((row * 3 + col // 8, 0, offset & ref.MASK, offset >> 32), (seed & ref.MASK, seed >> 32))
            bits = w[col % 8 // 2] >> (16 * (col % 2)) & 0xFFFF
            assert (f[row, col] != 0) == (bits >= ref.threshold(0.3))
    assert abs(float((ref.factor(64, 4096, 0.25, (1, 2)) == 0).double().mean()) - 0.25) < 5 * (0.25 * 0.75 / 2 ** 18) ** 0.5
    assert float(ref.factor(3, 9, 1.0, (1, 2)).abs().max()) == 0


@pytest.mark.parametrize("after", [None, "rms", "layer"])
@pytest.mark.parametrize("before", [None, "rms", "layer"])
def test_gradients_against_differences(after, before):
    """In 64 bits, central differences of the forward formulas."""
    torch.manual_seed(3)
    t, n, h = 3, 11, 1e-6
    make = lambda *s: torch.randn(s, dtype=torch.float64)  # noqa: E731
    norm = lambda k: None if k is None else Norm(make(n), make(n), kind=k, eps=1e-3)  # noqa: E731
    a, b = norm(after), norm(before)
    v = {"branch": make(t, n), "residual": make(t, n), "gate": make(n)}
    ds, dh = make(t, n), make(t, n)
    scale, p, rng = 0.75, 0.3, (1, 2)
    ref_rounded, ref.rounded = ref.rounded, lambda v, e, dt: e
    try:
        def loss():
            o = ref.join(v["branch"], v["residual"], a, b, v["gate"], scale, p, rng)
            return float((o["stream"][0] * ds).sum() + ((o["h"][0] * dh).sum() if b is not None else 0.0))
        stream = ref.join(v["branch"], v["residual"], a, b, v["gate"], scale, p, rng)["stream"][0]
        got = ref.join_backward(ds, dh if b is not None else None, v["branch"], stream, a, b, v["gate"], scale, p, rng)
        leaves = dict(v)
        for name, m in (("after", a), ("before", b)):
            if m is not None:
                leaves |= {f"{name}_weight": m.weight, f"{name}_bias": m.bias}
        for name, leaf in leaves.items():
            flat, want = leaf.view(-1), got[name][0].reshape(-1)
            for i in range(0, flat.numel(), 3):
                x = float(flat[i])
                flat[i] = x + h
                up = loss()
                flat[i] = x - h
                down = loss()
                flat[i] = x
                # (differences are off by the third derivative times h^2 and by 2^-53 of the loss over h)
                assert abs((up - down) / (2 * h) - float(want[i])) < 1e-6 * (1 + abs(float(want[i]))), (name, i)
        assert np.isfinite(loss())
    finally:
        ref.rounded = ref_rounded
