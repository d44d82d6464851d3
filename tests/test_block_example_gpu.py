"""The selective block's example: it learns its task, and what it serves token by token
after right-padded prompts is what the whole sequence gives."""
from __future__ import annotations

import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_trains_and_serves():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import selective_block

    first, last, worst = selective_block.run()
    assert last < 0.5 * first
    # float32 on both sides, outputs of order 1 to 10: 2^-24 x about 100 roundings x 10
    assert worst < 1e-4
