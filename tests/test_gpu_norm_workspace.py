"""Gradients of norms do not depend on what the workspace held (GPU)."""
import pytest
import torch

import paper_2506_01352_amd as tahq
from test_gpu_norm import ALPHA, EPS, KINDS, SHAPES, _cuda, _gates, _tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, cols", SHAPES + [(777, 1600), (2331, 160)])
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("halves", ("both", "post", "pre"))
def test_column_sums_are_all_written_before_they_are_read(rows, cols, kind, halves):
    """A workspace of NaN gives the bits that a workspace of zeros gives."""
    for gate_rows in _gates(rows, halves):
        d = _cuda(_tensors(rows, cols, gate_rows, halves, kind))
        cfg = tahq.make_norm_config(rows, cols, KINDS[kind][0], gate_rows, EPS, ALPHA)
        stats = torch.rand(2, rows, device="cuda") + 0.5
        need, got = tahq.tahq_norm_workspace_size(cfg), []
        for fill in (0x00, 0xFF):
            ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
            gr, gb, gg = torch.empty_like(d["grad_residual_out"]), None, None
            gw = {w: torch.empty(cols, device="cuda") for w in ("w_post", "w_pre") if d[w] is not None}
            if halves != "pre":
                gb = torch.empty_like(gr)
                gg = torch.empty_like(d["gate"], dtype=torch.float32) if gate_rows else None
            tahq.tahq_norm_backward(cfg, d["grad_residual_out"], d["grad_h"], d["block"], d["w_post"], d["gate"],
                                    d["residual"] if halves != "post" else None, d["w_pre"], stats, gr, gb, gw.get("w_post"), gg, gw.get("w_pre"), ws)
            got.append([v for v in (gr, gb, gg, *gw.values()) if v is not None])
        torch.cuda.synchronize()
        for a, b in zip(*got):
            assert torch.equal(a, b) and a.isfinite().all(), gate_rows
