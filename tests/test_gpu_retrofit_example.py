"""The retrofitting example: a few hundred steps teach it, and its compressed cache serves it."""
import math
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_taught_and_served(cuda_dev):
    import retrofit as example

    model, first, last, kept = example.train(150, 2.0, cuda_dev, quiet=True)
    assert math.isfinite(last) and last < 0.7 * first, (first, last)
    assert kept < 0.75, kept
    loss, slots = example.serve(model, cuda_dev)
    assert math.isfinite(loss) and loss < first, (first, loss)
    assert 0.0 < slots <= 1.0
