"""Calls whose launch would have 2^32 lanes or more, which the runtime does not take: refused before anything is enqueued (CPU)."""
import ctypes as C

import pytest

import paper_2506_01352_amd as tahq
from paper_2506_01352_amd import binding

P, BIG = 4096, 1 << 60                       # an aligned address that is never read
UNSUPPORTED = 3


def _status(name, *arguments):
    return getattr(binding._load(), name)(*[C.byref(a) if isinstance(a, C.Structure) else a for a in arguments])


@pytest.mark.parametrize("rows, cols", [(1 << 29, 8), ((1 << 29) - 31, 256), ((1 << 31) - 1, 1), (1 << 21, (1 << 16) - 255 + (1 << 16)), (1 << 20, 1 << 20)])
def test_matrices_of_more_tiles_than_a_launch_has_lanes_for(rows, cols):
    for dtype in (tahq.F32, tahq.BF16):
        cfg = tahq.make_mx4_config(rows, cols, dtype)
        assert _status("tahq_mx4_quantize", cfg, P, P, BIG, None, 0, None) == UNSUPPORTED
        assert _status("tahq_mx4_quantize", cfg, P, None, 0, P, BIG, None) == UNSUPPORTED
        assert _status("tahq_mx4_dequantize", cfg, P, BIG, P, None) == UNSUPPORTED


@pytest.mark.parametrize("m, n, k", [(1, 1 << 27, 64), (16, (1 << 27) - 15, 64), (1, (1 << 31) - 1, 64), ((1 << 31) - 1, (1 << 31) - 1, 64),
                                     (1 << 20, 1 << 28, 256)])
def test_products_of_more_tiles_than_a_launch_has_lanes_for(m, n, k):
    cfg = tahq.make_mx4_matmul_config(m, n, k, tahq.BF16)
    assert _status("tahq_mx4_matmul", cfg, P, BIG, P, BIG, P, P, BIG, None) == UNSUPPORTED
    x = tahq.make_mx4_config(m, k, tahq.BF16)
    assert _status("tahq_mx4_linear", x, cfg, P, P, BIG, P, P, BIG, None) == UNSUPPORTED


def test_a_layers_quantizer_is_refused_with_its_product_and_the_other_way_round():
    """Whichever of the two launches does not go, neither is enqueued."""
    rows = (1 << 29) + 1
    for m, n, k in ((rows, 64, 8), (16, 1 << 28, 64)):
        x, cfg = tahq.make_mx4_config(m, k, tahq.BF16), tahq.make_mx4_matmul_config(m, n, k, tahq.BF16)
        assert _status("tahq_mx4_linear", x, cfg, P, P, BIG, P, P, BIG, None) == UNSUPPORTED
