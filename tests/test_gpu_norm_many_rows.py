"""Norms of more rows than a launch has wavefronts for (GPU)."""
import pytest
import torch

import paper_2506_01352_amd as tahq

pytestmark = pytest.mark.gpu

UNIT, EPS = 2.0 ** -24, 1e-6


@pytest.mark.parametrize("rows", ((1 << 27) + 5, 1 << 26))
def test_forward_of_very_many_short_rows(rows):
    """Both sides of the limit at two rows to a workgroup; h within the roundings of a sum of three squares and a quotient, packed h the
    quantizer's of it."""
    cols = 3
    g = torch.Generator(device="cuda").manual_seed(2)
    r = torch.randn(rows, cols, generator=g, device="cuda")
    w = torch.tensor([0.5, -1.25, 2.0], device="cuda")
    out, h = torch.empty_like(r), torch.full((rows + 1, cols), 7.0, device="cuda")
    stats = torch.empty(2, rows, device="cuda")
    size = tahq.tahq_mx4_packed_size(rows, cols)
    packed = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    cfg = tahq.make_norm_config(rows, cols, tahq.F32, 0, EPS, 1.0, 0, 0, tahq.MX4_COVER)
    tahq.tahq_norm_forward(cfg, r, None, None, None, w, out, h, packed, stats)
    torch.cuda.synchronize()
    assert torch.equal(out, r) and (h[rows] == 7.0).all() and (packed[size:] == 0xA5).all() and (stats[0] == 0).all()
    for at in range(0, rows, 1 << 24):
        x = r[at:at + (1 << 24)].double()
        rstd = (x.square().mean(1) + EPS).rsqrt()
        want = x * rstd[:, None] * w.double()
        assert ((stats[1, at:at + (1 << 24)].double() - rstd).abs() <= 64 * UNIT * rstd).all()
        assert ((h[at:min(at + (1 << 24), rows)].double() - want).abs() <= 64 * UNIT * want.abs() + 1e-38).all()
    again = torch.empty(size, dtype=torch.uint8, device="cuda")
    tahq.tahq_mx4_quantize(tahq.make_mx4_config(rows, cols, tahq.F32, 0, 0, tahq.MX4_COVER), h, again)
    assert torch.equal(packed[:size], again)
