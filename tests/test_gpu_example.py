"""The example: a gated block trained with 8-bit checkpoints and served from 4-bit weights."""
import importlib.util
import os

import pytest

from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


def test_gated_block_learns_and_is_served():
    need_gpu()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    first, last, error = m.run(tokens=200, width=136, hidden=360, steps=60, served=3, say=say)
    assert last < 0.7 * first
    # a 4-bit weight is off by a tenth of its size; three products of them and a gate
    assert error < 0.35
