"""The example that trains and serves with the token mixers."""
import os
import sys

import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def test_example_learns_and_serves():
    """The model learns to repeat (from log 32 and more to a small part of it), and the logits served from the cache and the
    state are the whole forward's.  Both paths round the same values to bf16 in other
    orders: three such roundings (2^-8 each) of sums of size about 1 pass two matrices,
    and logits are of size up to some ten."""
    require_gpu()
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_mixers
    first, last, off = token_mixers.main(quiet=True)
    assert last < 0.2 * first
    assert off < 0.3, off
