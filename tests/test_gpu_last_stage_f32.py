"""The last stage's step (examples/last_stage.py) in fp32, whose roundings are small enough to show a token, a tile or a small term that is missing, and with the
dropout's mask from its definition instead of from the library."""
import os
import sys

import pytest
import torch

from oracle import dropout

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu

SIZES = [dict(batch=2, seq=96, hidden=512, heads=8, k_heads=2, vocab=5003), dict(batch=3, seq=65, hidden=320, heads=5, k_heads=5, vocab=1000),
         dict(batch=4, seq=150, hidden=576, heads=6, k_heads=2, vocab=16001)]
UNIT = 2.0 ** -24


def _kept(sizes, seed=3):
    import last_stage
    n = sizes["batch"] * sizes["seq"] * sizes["hidden"]
    return torch.from_numpy(dropout.kept(0, n, last_stage.P, seed, 0))


@pytest.mark.parametrize("sizes", SIZES)
def test_gradients_of_a_step_in_fp32(sizes):
    """Between the received activations and any gradient lie about sixteen tensors, each stored in fp32 and made by a sum of K terms at the most, which is off by sqrt(K) roundings of
    the terms' norm as if these were drawn; all as if added up the same way.  The loss is off by those of the six in front of it, of which logits of size 4 and less make as much."""
    import last_stage
    got = last_stage.run(**sizes, dtype="f32", mask=_kept(sizes))
    each = (1 + max(sizes["vocab"], sizes["hidden"], sizes["batch"] * sizes["seq"]) ** 0.5) * UNIT
    assert abs(got["loss"] - got["loss64"]) < 6 * 4 * each
    bad = {n: e for n, e in got["errors"].items() if not e < 16 * each}
    assert not bad, (16 * each, got["errors"])


@pytest.mark.parametrize("sizes", SIZES)
def test_gradients_of_a_step_with_the_mask_of_its_definition(sizes):
    """bf16: the bounds of test_gpu_last_stage.py."""
    import last_stage
    got = last_stage.run(**sizes, mask=_kept(sizes))
    assert abs(got["loss"] - got["loss64"]) < 6 * 4 * 2.0 ** -8
    bad = {n: e for n, e in got["errors"].items() if not e < 16 * 2.0 ** -8}
    assert not bad, got["errors"]


def test_a_mask_of_another_seed_shows():
    import last_stage
    got = last_stage.run(**SIZES[1], dtype="f32", mask=_kept(SIZES[1], seed=4))
    assert got["errors"]["w_o"] > 0.05
