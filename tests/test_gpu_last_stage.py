"""Heads, dropout and loss together with codec and norms, as a last pipeline stage runs them (examples/last_stage.py)."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [dict(batch=2, seq=96, hidden=512, heads=8, k_heads=2, vocab=5003), dict(batch=3, seq=65, hidden=320, heads=5, k_heads=5, vocab=1000)])
def test_gradients_of_a_step(sizes):
    """Between the received activations and any gradient lie about sixteen tensors stored in bf16, each off by 2^-8 at the most and all as if added up the
    same way; the loss is a mean over tokens, off by the roundings of the six in front of it, of which logits of size 4 and less make as much."""
    import last_stage
    got = last_stage.run(**sizes)
    assert abs(got["loss"] - got["loss64"]) < 6 * 4 * 2.0 ** -8
    bad = {n: e for n, e in got["errors"].items() if not e < 16 * 2.0 ** -8}
    assert not bad, got["errors"]
