"""The example layer runs and stays near the fp32 layer: 8 bits for rows and weights in two products in a row.

Tolerance, before the first run: a code of a row (or channel) whose largest value is about 3.5 times its rms stands for a
value within half a step: int8 0.5 * 3.5 / 127 / sqrt(3) = 0.8 % of the rms, e4m3 at most 2^-4 / sqrt(3) = 3.6 % of each
value.  A product's error adds the row's and the channel's: sqrt(2) times that; three products (gate and up enter the
same factor) and their roundings stay below four times the single error: 3.2 % and 14.4 %."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("kind,limit", [("int8", 0.032), ("e4m3", 0.144)])
@pytest.mark.parametrize("size", [["--tokens", "1", "--ranks", "1", "--hidden", "256", "--inner", "128"],
                                  ["--tokens", "77", "--hidden", "528", "--inner", "208", "--experts", "8", "--topk", "2"],
                                  ["--tokens", "300"]])
def test_example_layer(kind, limit, size):
    import moe_layer
    assert moe_layer.main(size + ["--kind", kind, "--steps", "2"]) < limit
