"""The classes' state: streams, what is kept from the forward pass for the backward one, refusals (GPU)."""
import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import norm64

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -24           # half a unit in the last place of an fp32 number


def _np(v):
    return v.double().cpu().numpy()


@pytest.mark.parametrize("accumulate", (0, 1))
def test_norms_on_a_stream_of_their_own_from_the_first_call_on(accumulate):
    """Forward and twice backward on a side stream; within 128 roundings of the terms' magnitudes, and one for every row of a sum."""
    rows, cols, gate_rows, eps, alpha = 3000, 1600, 700, 1e-6, 0.8125
    g = torch.Generator().manual_seed(6)
    t = {n: torch.randn(rows, cols, generator=g) for n in ("residual", "block", "grad_out", "grad_h")}
    t.update(w_post=1 + 0.2 * torch.randn(cols, generator=g), w_pre=1 + 0.2 * torch.randn(cols, generator=g), gate=torch.randn(5, cols, generator=g))
    d = {n: v.cuda() for n, v in t.items()}
    norm = tahq.BlockNorm(tahq.make_norm_config(rows, cols, tahq.F32, gate_rows, eps, alpha, accumulate))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, _ = norm.forward(d["residual"], d["block"], d["w_post"], d["gate"], d["w_pre"], stream=side)
    for _ in range(2):
        got = norm.backward(d["grad_out"], d["grad_h"], d["block"], d["w_post"], d["gate"], out, d["w_pre"], norm.stats, stream=side)
    side.synchronize()
    n = {k: v.double().numpy() for k, v in t.items()}
    want = norm64.backward(n["grad_out"], n["grad_h"], n["block"], n["w_post"], n["gate"], _np(out), n["w_pre"], *_np(norm.stats), gate_rows, alpha)
    for name in ("grad_residual", "grad_block", "grad_w_post", "grad_gate", "grad_w_pre"):
        sums = name not in ("grad_residual", "grad_block")
        times = 1 + accumulate if sums else 1
        off = (128 + (rows if sums else 0)) * UNIT * times * want[name + "_size"] + 1e-38
        assert (np.abs(_np(got[name]) - times * want[name]) <= off).all(), name


def test_training_through_an_h_that_is_packed_already():
    """x given along channels and along tokens: the same bits as of a forward pass that packs it, whatever x came before."""
    tokens, n, k = 200, 300, 1600
    w, x, other, dy = (torch.randn(*s, device="cuda").to(torch.bfloat16) for s in ((n, k), (tokens, k), (tokens, k), (tokens, n)))
    layer = tahq.Mx4Linear(w, tokens, transform=1, scale_rule=tahq.MX4_COVER, training=True)
    y = layer.forward(x).clone()
    dx, dw = (t.clone() for t in layer.backward(dy))
    packed = tahq.Mx4Tensor(tahq.make_mx4_config(tokens, k, tahq.BF16, 0, 1, tahq.MX4_COVER), transposed=True)
    packed.quantize(x)
    layer.forward(other)
    assert torch.equal(layer.product(packed.packed, x_packed_t=packed.packed_t), y)
    got = layer.backward(dy)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)


def test_two_micro_batches_in_flight_give_what_they_give_one_after_the_other():
    rows, cols, n = 100, 512, 320
    g = torch.Generator(device="cuda").manual_seed(9)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    w, w_post, w_pre, gate = make(n, cols), make(cols), make(cols), make(1, cols)
    batches = [{"residual": make(rows, cols), "block": make(rows, cols), "dy": make(rows, n), "dr": make(rows, cols)} for _ in range(2)]
    cfg = tahq.make_norm_config(rows, cols, tahq.BF16, rows)

    def forward(norm, layer, b, slot):
        out, h = norm.forward(b["residual"], b["block"], w_post, gate, w_pre, slot=slot)
        return out, layer.forward(h, slot=slot)

    def backward(norm, layer, b, out, slot):
        dh, dw = layer.backward(b["dy"], slot=slot)
        got = norm.backward(b["dr"], dh, b["block"], w_post, gate, out, w_pre, norm.stats_of(slot))
        return [t.clone() for t in (dw, *got.values())]

    one, one_layer = tahq.BlockNorm(cfg), tahq.Mx4Linear(w, rows, training=True)
    want, ys = [], []
    for b in batches:
        out, y = forward(one, one_layer, b, 0)
        ys.append(y.clone())
        want.append(backward(one, one_layer, b, out, 0))
    both, both_layer = tahq.BlockNorm(cfg, in_flight=2), tahq.Mx4Linear(w, rows, training=True, in_flight=2)
    kept = [forward(both, both_layer, b, i) for i, b in enumerate(batches)]
    for i, b in enumerate(batches):
        assert torch.equal(kept[i][1], ys[i])
        assert all(torch.equal(a, c) for a, c in zip(backward(both, both_layer, b, kept[i][0], i), want[i]))
