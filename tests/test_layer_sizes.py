"""Sizes at and past the dense layer operators' limits (CPU only)."""
import pytest
import torch

from paper_2608_16308_amd import Checkpoint, DbsError, layer
from paper_2608_16308_amd._lib import DBS_ERR_UNSUPPORTED

META = torch.device("meta")
BF = torch.bfloat16


def test_sizes_that_do_not_fit_the_abi():
    """2^32 + 3 rows must not arrive as 3 (meta tensors have no memory)."""
    for shape in (((1 << 32) + 3, 1), (1, (1 << 32) + 3), ((1 << 31) + 1, 2), ((1 << 30) + 1, 1)):
        t = torch.empty(shape, dtype=BF, device=META)
        with pytest.raises(DbsError) as e:
            layer.check_rows(t, "x", BF, META, None, None)
        assert e.value.status == DBS_ERR_UNSUPPORTED
        c = Checkpoint(torch.empty(shape, dtype=torch.int8, device=META),
                       torch.empty((shape[0], -(-shape[1] // 32)), dtype=torch.uint8, device=META), BF)
        with pytest.raises(DbsError) as e:
            layer.check_checkpoint(torch, c, "c", BF, META, *shape)
        assert e.value.status == DBS_ERR_UNSUPPORTED
    for shape in ((1 << 30, 1), (1, 1 << 30)):
        layer.check_rows(torch.empty(shape, dtype=BF, device=META), "x", BF, META, None, None)
