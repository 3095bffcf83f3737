"""The layer context's part of the C ABI (CPU only)."""
import os

import paper_2608_16308_amd as dbs
from paper_2608_16308_amd import _lib

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dbspmspv.h")


def test_a_context_keeps_its_stream():
    """Its workspace holds sums between two kernels of a call: another stream
    would write them while they are read."""
    name = "dbs_layer_set_stream"
    assert name not in _lib.EXPORTED and not hasattr(dbs.lib(), name)
    with open(HEADER) as f:
        assert name not in f.read()
