"""Norms of tensors that take paths of their own by size: eight rows to a workgroup forward, teams of workgroups backward (GPU)."""
import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import mx4, norm64
from test_gpu_norm import ALPHA, EPS, HALF, KINDS, UNIT, _cuda, _np, _tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, cols, gate_rows", [(2049, 6152, 700), (2115, 6157, 1), (2048, 8192, 0)])
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("transform, rule", [(0, tahq.MX4_FLOOR), (1, tahq.MX4_COVER)])
def test_forward_with_eight_rows_to_a_workgroup(rows, cols, gate_rows, kind, transform, rule):
    """h, r' and statistics within the bounds of test_gpu_norm's forward pass; the packed h is the quantizer's of the fp32 h."""
    t = _tensors(rows, cols, gate_rows, "both", kind)
    d = _cuda(t)
    wide = {n: None if v is None else v.float() for n, v in d.items()}
    packed, results = [], []
    for dtype, x in ((KINDS[kind][0], d), (tahq.F32, wide)):
        cfg = tahq.make_norm_config(rows, cols, dtype, gate_rows, EPS, ALPHA, 0, transform, rule)
        p = torch.full((tahq.tahq_mx4_packed_size(rows, cols) + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        out, h, stats = torch.full_like(x["residual"], 7.0), torch.full_like(x["residual"], 7.0), torch.full((2, rows), 7.0, device="cuda")
        tahq.tahq_norm_forward(cfg, x["residual"], x["block"], x["w_post"], x["gate"], x["w_pre"], out, h, p, stats)
        packed.append(p.cpu().numpy())
        results.append((out, h, stats))
    want_packed = mx4.quantize(results[1][1].cpu().numpy(), transform, rule)
    for p in packed:
        assert (p[want_packed.size:] == 0xA5).all() and (p[:want_packed.size] == want_packed).all()
    out, h, stats = (_np(v) for v in results[0])
    n = {k: _np(v) for k, v in t.items()}
    want, want_h, rb, rr = norm64.forward(n["residual"], n["block"], n["w_post"], n["gate"], n["w_pre"], gate_rows, float(np.float32(EPS)), ALPHA)
    size = np.abs(ALPHA * n["residual"])
    size = size + np.abs(want - ALPHA * n["residual"])
    assert (np.abs(out - want) <= 64 * UNIT * size + HALF[kind] * np.abs(want) + 1e-38).all()
    spread = np.sqrt((np.square(size).mean(1) + EPS) / (np.square(want).mean(1) + EPS))
    assert (np.abs(stats[0] - rb) <= 64 * UNIT * rb).all() and (np.abs(stats[1] - rr) <= 192 * UNIT * rr * spread).all()
    off = (256 * UNIT * spread[:, None] * (np.abs(want_h) + np.abs(size * rr[:, None] * n["w_pre"]))) + HALF[kind] * np.abs(want_h) + 1e-38
    assert (np.abs(h - want_h) <= off).all()


@pytest.mark.parametrize("rows, cols, gate_rows, kind, halves", [
    (23000, 1024, 23000, "bf16", "both"), (23000, 1024, 0, "bf16", "post"), (23000, 1024, 0, "bf16", "pre"), (23000, 1024, 700, "bf16", "post"),
    (9001, 2500, 9001, "bf16", "both"), (11300, 1000, 400, "f32", "post"), (11300, 1000, 0, "f32", "pre"), (4600, 5120, 1024, "bf16", "both"),
    (2900, 8192, 500, "bf16", "both"), (45000, 512, 21, "bf16", "both")])
@pytest.mark.parametrize("accumulate", (0, 1))
def test_backward_by_teams_of_workgroups(rows, cols, gate_rows, kind, halves, accumulate):
    """The six tensors are past the last cache; as test_gpu_norm's backward pass."""
    assert rows * cols * 6 * (2 if kind == "bf16" else 4) >= 256 << 20
    t = _tensors(rows, cols, gate_rows, halves, kind)
    n = {k: _np(v) for k, v in t.items()}
    out, _, rb, rr = norm64.forward(n["residual"], n["block"], n["w_post"], n["gate"], n["w_pre"], gate_rows, EPS, ALPHA)
    t["residual_out"] = torch.from_numpy(out).to(KINDS[kind][1]) if halves != "post" else None
    stats = torch.from_numpy(np.stack((rb, rr))).float()
    want = norm64.backward(n["grad_residual_out"], n["grad_h"], n["block"], n["w_post"], n["gate"], _np(t["residual_out"]), n["w_pre"],
                           *stats.double().numpy(), gate_rows, ALPHA)
    d = _cuda(t)
    cfg = tahq.make_norm_config(rows, cols, KINDS[kind][0], gate_rows, EPS, ALPHA, accumulate)
    got = {"grad_residual": torch.full((rows, cols), 7.0, dtype=KINDS[kind][1], device="cuda")}
    if halves != "pre":
        got["grad_block"], got["grad_w_post"] = torch.full_like(got["grad_residual"], 7.0), torch.full((cols,), 0.5, device="cuda")
    if d["gate"] is not None:
        got["grad_gate"] = torch.full_like(d["gate"], 0.5, dtype=torch.float32)
    if halves != "post":
        got["grad_w_pre"] = torch.full((cols,), 0.5, device="cuda")
    need = tahq.tahq_norm_workspace_size(cfg)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN in what is not written
    tahq.tahq_norm_backward(cfg, d["grad_residual_out"], d["grad_h"], d["block"], d["w_post"], d["gate"], d["residual_out"], d["w_pre"],
                            stats.cuda(), got["grad_residual"], got.get("grad_block"), got.get("grad_w_post"), got.get("grad_gate"),
                            got.get("grad_w_pre"), ws)
    torch.cuda.synchronize()
    assert (ws[need:] == 0xFF).all()
    for name, g in got.items():
        w, size, small = want[name], want[name + "_size"], name in ("grad_residual", "grad_block")
        before = 0.5 if accumulate and not small else 0.0
        off = (128 + (0 if small else rows)) * UNIT * (size + before) + (HALF[kind] * np.abs(w) if small else 0) + 1e-38
        assert (np.abs(_np(g) - (w + before)) <= off).all(), name
