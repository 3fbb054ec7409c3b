"""The example that runs convolution, group norm, 4-bit rows, 4-bit linear layer and the norm's gradient together."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_bottleneck_example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import bottleneck_4bit
    r = bottleneck_4bit.main()
    # two operands held in 4 bits, each with a relative error of about 0.1 (a uniform error of half a step, steps of 1/6 to 1/2 of a value)
    assert 0.01 < r["error"] < 0.3
    assert r["losses"][-1] < 0.2 * r["losses"][0]
    assert r["values"].isfinite().all()
