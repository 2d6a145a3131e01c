"""A step over a stage boundary, codec, norms and mx4 products together (examples/mx4_stage.py)."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [dict(batch=2, seq=96, hidden=512, features=300), dict(batch=3, seq=65, hidden=1600, features=513)])
def test_a_step_stays_near_the_unquantized_one(sizes):
    """4-bit floating point is off by up to an eighth of a value between grid points and 3.8-bit tiles by about as much; three of them in a row, added as
    squares, give 0.3 at the most.  What is not quantized is off by bf16's roundings."""
    import mx4_stage
    got = mx4_stage.run(**sizes)
    assert got["errors"]["r'"] < 2.0 ** -8
    assert got["activation bytes"] < 0.35 * got["bf16 bytes"] and got["gradient bytes"] < 0.51 * got["bf16 bytes"]
    bad = {n: e for n, e in got["errors"].items() if not e < 0.3}
    assert not bad, got["errors"]
