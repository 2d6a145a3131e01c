"""Rows and columns that fill up a packed h are zeros with scale byte 0, whatever the rows and weights hold (GPU)."""
import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import mx4

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.mark.parametrize("rows, cols", [(1, 40), (33, 65), (45, 250), (40, 257), (5, 1600), (70, 2000)])
@pytest.mark.parametrize("kind", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("transform", (0, 1))
@pytest.mark.parametrize("halves", ("both", "pre"))
@pytest.mark.parametrize("spoiled", ("negative weight", "infinite weight", "NaN weight", "NaN row", "infinite row"))
def test_padding_of_a_packed_h_is_zeros(rows, cols, kind, transform, halves, spoiled):
    """Byte for byte the quantizer's matrix of the same fp32 h, whose padding is written on its own."""
    g = torch.Generator().manual_seed(rows + cols)
    make = lambda *s: torch.randn(*s, generator=g)      # noqa: E731
    t = {"residual": make(rows, cols), "block": make(rows, cols), "w_post": make(cols), "gate": make(rows, cols), "w_pre": make(cols)}
    t["w_pre"][cols - 1] = -1.0
    if spoiled.endswith("weight"):
        t["w_pre"][cols // 2] = {"negative": -2.0, "infinite": float("inf"), "NaN": float("nan")}[spoiled.split()[0]]
    else:
        t["block" if halves == "both" else "residual"][rows // 2, cols // 3] = float("nan" if spoiled.startswith("NaN") else "inf")
    if halves == "pre":
        t.update(block=None, w_post=None, gate=None)
    t = {n: None if v is None else v.to(kind).float().cuda() for n, v in t.items()}       # what the type holds, in either type
    size = tahq.tahq_mx4_packed_size(rows, cols)
    packed = {}
    for dtype, torch_dtype in ((tahq.F32, torch.float32), (tahq.BF16, torch.bfloat16)):
        if kind is torch.float32 and dtype == tahq.BF16:
            continue
        d = {n: None if v is None else v.to(torch_dtype) for n, v in t.items()}
        # a negative scale turns zeros behind the columns into negative zeros
        cfg = tahq.make_norm_config(rows, cols, dtype, 1 if halves == "both" else 0, EPS, -0.75, 0, transform, tahq.MX4_COVER)
        out = torch.empty_like(d["residual"])
        h = torch.empty_like(out) if dtype == tahq.F32 else None
        packed[dtype] = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
        tahq.tahq_norm_forward(cfg, d["residual"], d["block"], d["w_post"], d["gate"], d["w_pre"], out, h, packed[dtype], None)
        if h is not None:
            want = mx4.quantize(h.cpu().numpy(), transform, mx4.COVER)
    for p in packed.values():
        bad = np.flatnonzero(p.cpu().numpy() != want)
        assert bad.size == 0, f"{bad.size} bytes differ, first at {bad[0]}"
