"""Dropout through the C ABI: every element against the mask's definition, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import dropout

pytestmark = pytest.mark.gpu

KINDS = {"f32": (tahq.F32, torch.float32), "bf16": (tahq.BF16, torch.bfloat16)}


def _want(x, residual, p, seed, offset, kind):
    """fp32 products and sums, rounded once: exact in NumPy's fp32, and torch rounds to bf16 like the kernel."""
    kept = torch.from_numpy(dropout.kept(0, x.numel(), p, seed, offset))
    y = torch.where(kept, x.float().flatten() * float(dropout.scale(p)), torch.zeros(()))
    if residual is not None:
        y = residual.float().flatten() + y
    return y.to(KINDS[kind][1])


def _same(a, b):
    """Bit for bit; NaN is NaN."""
    a, b = a.float(), b.float()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(nan=1.0), b.nan_to_num(nan=1.0))


@pytest.mark.parametrize("elements", (1, 2, 7, 8, 9, 63, 64, 65, 511, 2047, 2048, 2049, 100003))
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("p, seed, offset", [(0.1, 0, 0), (0.5, 0xFEDCBA9876543210, (1 << 64) - 1), (0.0, 3, 4), (1.0, 5, 6), (0.9999, 7, 1 << 40)])
def test_every_element(elements, kind, p, seed, offset):
    g = torch.Generator().manual_seed(elements)
    x, residual = (torch.randn(elements, generator=g).to(KINDS[kind][1]) for _ in range(2))
    if elements > 8:
        x[3], x[5] = float("nan"), float("inf")
    cfg = tahq.make_dropout_config(elements, KINDS[kind][0], p, seed, offset)
    for r in (None, residual):
        out = torch.full((elements + 16,), 7.0, dtype=KINDS[kind][1], device="cuda")
        tahq.tahq_dropout_forward(cfg, x.cuda(), None if r is None else r.cuda(), out)
        torch.cuda.synchronize()
        assert _same(out[:elements].cpu(), _want(x, r, p, seed, offset, kind)) and (out[elements:] == 7).all()
    grad = torch.full((elements + 16,), 7.0, dtype=KINDS[kind][1], device="cuda")
    tahq.tahq_dropout_backward(cfg, x.cuda(), grad)
    assert _same(grad[:elements].cpu(), _want(x, None, p, seed, offset, kind)) and (grad[elements:] == 7).all()


def test_places_far_behind():
    """More elements than 32 bits count, and a tensor of which the first and last are looked at."""
    n = (1 << 32) + (1 << 20) + 5
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    tahq.tahq_dropout_backward(tahq.make_dropout_config(n, tahq.BF16, 0.5, 11, 2), x, x)
    for first in (0, (1 << 32) - 4096, (1 << 32) + 77, n - 1000):
        assert torch.equal(x[first:first + 1000].cpu().float() != 0, torch.from_numpy(dropout.kept(first, 1000, 0.5, 11, 2)))


def test_in_place():
    x, r = torch.randn(1000, device="cuda"), torch.randn(1000, device="cuda")
    cfg = tahq.make_dropout_config(1000, tahq.F32, 0.3, 9, 1)
    want = _want(x.cpu(), r.cpu(), 0.3, 9, 1, "f32")
    a, b = x.clone(), r.clone()
    tahq.tahq_dropout_forward(cfg, a, r, a)
    tahq.tahq_dropout_forward(cfg, x, b, b)
    assert torch.equal(a.cpu(), want) and torch.equal(b.cpu(), want)


def test_class_counts_and_keeps_offsets():
    drop = tahq.Dropout(tahq.make_dropout_config(4 * 33, tahq.F32, 0.5, 21, 100), in_flight=2)
    x = torch.randn(4, 33, device="cuda")
    ones = torch.ones_like(x)
    outs = [drop.forward(x, slot=i).clone() for i in (0, 1, 0)]
    assert outs[0].shape == x.shape
    for out, offset in zip(outs, (100, 101, 102)):
        assert torch.equal(out.flatten().cpu(), _want(x.cpu(), None, 0.5, 21, offset, "f32"))
    for slot, offset in ((1, 101), (0, 102)):
        assert torch.equal((drop.backward(ones, slot=slot) != 0).flatten().cpu(), torch.from_numpy(dropout.kept(0, x.numel(), 0.5, 21, offset)))
    with pytest.raises(ValueError):
        tahq.Dropout(tahq.make_dropout_config(8, tahq.F32, 0.5)).backward(torch.ones(8, device="cuda"))
    with pytest.raises(ValueError):
        drop.forward(x, torch.randn(33, 4, device="cuda"))
    for bad in (x.bfloat16(), x[:, :32], x.cpu(), torch.randn(33, 4, device="cuda").t()):
        with pytest.raises((ValueError, AssertionError)):
            drop.forward(bad)


def test_graph_replays_take_other_masks():
    """A captured pass and its backward pass, replayed with another number in the offset, eager work in between."""
    more = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = tahq.Dropout(tahq.make_dropout_config(5000, tahq.BF16, 0.25, 1, 50), graph_offset=more)
    x, r = (torch.randn(5000, device="cuda").bfloat16() for _ in range(2))
    drop.forward(x, r, offset=50)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = drop.forward(x, r, offset=50)
        grad = drop.backward(r)
    eager = tahq.Dropout(tahq.make_dropout_config(5000, tahq.BF16, 0.25, 1))
    for replay in range(4):
        more.fill_(replay * 3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager.forward(x, r, offset=50 + replay * 3)) and torch.equal(grad, eager.backward(r))
        assert _same(out.cpu(), _want(x.cpu(), r.cpu(), 0.25, 1, 50 + replay * 3, "bf16"))


def test_class_keeps_its_configuration():
    """What the caller does to the configuration afterwards changes nothing."""
    cfg = tahq.make_dropout_config(64, tahq.F32, 0.5, 3)
    drop = tahq.Dropout(cfg)
    x = torch.randn(64, device="cuda")
    want = drop.forward(x, offset=0).clone()
    cfg.elements, cfg.seed, cfg.p = 1 << 40, 9, 0.0
    assert torch.equal(drop.forward(x, offset=0), want)
