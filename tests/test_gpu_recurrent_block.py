"""The operators together: the example trains, and decodes what the scan computes."""
import os
import sys

import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_example_learns_and_decodes():
    """Leaky averages are within the reach of the block: the loss has to fall to a fifth of the first one at the least.  Decoding may differ
    from the scan by the order of its sums, which can move an 8-bit rounding of h by a code (1/16 of a term of a sum of 128)."""
    require_gpu()
    import recurrent_block
    first, last, off, size = recurrent_block.run(steps=150)
    assert last < 0.2 * first
    assert off <= 0.05 * size
