"""Host side of dropout, heads and loss: sizes, defaults, frequencies, refusals before anything is enqueued, and their oracles.  CPU only."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import dropout, heads64, loss64
from paper_2506_01352_amd import binding

P = 4096                                     # an aligned address that is never read: every call here is refused
BIG = 1 << 40


def _status(name, *arguments):
    return getattr(binding._load(), name)(*[C.byref(a) if isinstance(a, C.Structure) else a for a in arguments])


def test_defaults():
    d, h, r, c = (f() for f in (tahq.tahq_dropout_config_default, tahq.tahq_heads_config_default, tahq.tahq_rotary_config_default, tahq.tahq_loss_config_default))
    assert (d.struct_size, d.dtype, d.elements, d.seed, d.offset) == (C.sizeof(d), tahq.BF16, 0, 0, 0) and d.p == np.float32(0.1)
    assert (h.struct_size, h.dtype, h.norm, h.layout, h.tokens, h.magnitude) == (C.sizeof(h), tahq.BF16, 1, tahq.HEADS_HALVES, 0, 1.0)
    assert (r.struct_size, r.base, r.factor, r.original, r.low, r.high, r.scaling) == (C.sizeof(r), 10000.0, 1.0, 4096, 1.0, 32.0, tahq.ROTARY_PLAIN)
    assert (c.struct_size, c.dtype, c.weight_dtype, c.reduction, c.ignore, c.accumulate) == (C.sizeof(c), tahq.BF16, tahq.BF16, tahq.LOSS_MEAN, -100, 0)
    for name in ("dropout", "heads", "rotary", "loss"):
        getattr(binding._load(), f"tahq_{name}_config_default")(None)


# ---------------------------------------------------------------- dropout

def test_generator_is_the_published_one():
    """The published test vectors of Philox 4x32, ten rounds."""
    ones = 0xFFFFFFFF
    for counter, key, want in (((0,) * 4, (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                               ((ones,) * 4, (ones, ones), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                               ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(v) for v in dropout.philox(counter, key)) == want


def test_mask_keeps_its_share():
    """A share of n independent draws lies within six standard deviations."""
    n = 200000
    for p in (0.0, 0.1, 0.5, 0.9, 1.0):
        kept = dropout.kept(0, n, p, 1234567890123, 5)
        assert abs(kept.mean() - (1 - dropout.threshold(p) / 65536)) <= 6 * math.sqrt(p * (1 - p) / n)
    a, b = (dropout.kept(0, n, 0.5, 7, offset) for offset in (0, 1))
    assert abs((a == b).mean() - 0.5) <= 6 * 0.5 / math.sqrt(n)
    assert (dropout.kept(1000, 77, 0.5, 7, 0) == a[1000:1077]).all()


@pytest.mark.parametrize("field, value", [("elements", 0), ("elements", (1 << 48) + 1), ("dtype", 2), ("p", -0.1), ("p", 1.5), ("p", float("nan")), ("struct_size", 8)])
def test_dropout_refuses_configurations(field, value):
    cfg = tahq.make_dropout_config(64, tahq.BF16, 0.1)
    setattr(cfg, field, value)
    assert _status("tahq_dropout_forward", cfg, P, None, P, None, None) == 2 and _status("tahq_dropout_backward", cfg, P, P, None, None) == 2


def test_dropout_refuses_arguments():
    cfg = tahq.make_dropout_config(64, tahq.BF16, 0.1)
    f = lambda *a: _status("tahq_dropout_forward", cfg, *a, None)      # noqa: E731
    b = lambda *a: _status("tahq_dropout_backward", cfg, *a, None)     # noqa: E731
    assert f(None, P, P, None) == 1 and f(P, P, None, None) == 1 and b(None, P, None) == 1 and b(P, None, None) == 1
    assert f(P + 2, P, P, None) == 6 and f(P, P + 8, P, None) == 6 and f(P, P, P + 4, None) == 6 and f(P, P, P, P + 4) == 6 and b(P, P, P + 1) == 6
    assert _status("tahq_dropout_forward", None, P, P, P, None, None) == 1
    with pytest.raises(ValueError):
        tahq.tahq_dropout_forward(cfg, torch.zeros(64, dtype=torch.float32), None, torch.zeros(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        tahq.tahq_dropout_forward(cfg, torch.zeros(63, dtype=torch.bfloat16), None, torch.zeros(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        tahq.tahq_dropout_backward(cfg, torch.zeros(64, dtype=torch.float16), torch.zeros(64, dtype=torch.bfloat16))


# ---------------------------------------------------------------- heads

SCALINGS = {"plain": 0, "linear": 1, "stretched": 2, "parts": 3}


@pytest.mark.parametrize("rotated", (2, 4, 40, 64, 128, 512))
@pytest.mark.parametrize("scaling, factor", [("plain", 1.0), ("linear", 4.0), ("stretched", 8.0), ("parts", 8.0), ("parts", 3.7)])
def test_frequencies(rotated, scaling, factor):
    """The 64-bit formulas' frequencies, off by the roundings of a power in 64 bits: the exponent's, and ln(base) of it, which counts 20 times at the
    most, and a dozen more."""
    cfg = tahq.make_rotary_config(rotated, 10000.0, SCALINGS[scaling], factor)
    got = tahq.tahq_rotary_frequencies(cfg)
    want = heads64.frequencies(rotated, 10000.0, scaling, factor)
    assert len(got) == rotated // 2
    for g, w in zip(got, want):
        assert abs(g / 2.0 ** 64 * 2 * math.pi - w) <= 40 * 2.0 ** -53 * w + 2.0 ** -62


def test_stretched_ends():
    """The fastest pair keeps its frequency, the slowest one turns as much slower as the context is longer."""
    plain, stretched = (tahq.tahq_rotary_frequencies(tahq.make_rotary_config(128, 10000.0, s, 4.0)) for s in (tahq.ROTARY_PLAIN, tahq.ROTARY_STRETCHED))
    assert plain[0] == stretched[0] and abs(plain[-1] / stretched[-1] - 4.0) < 1e-9


@pytest.mark.parametrize("field, value", [("rotated", 0), ("rotated", 7), ("scaling", 4), ("base", 0.0), ("base", -1.0), ("base", float("nan")), ("factor", 0.0),
                                          ("factor", float("inf")), ("original", 0), ("low", 32.0), ("high", float("nan")), ("struct_size", 4)])
def test_frequencies_refuse(field, value):
    cfg = tahq.make_rotary_config(64, scaling=tahq.ROTARY_PARTS, factor=2.0)
    setattr(cfg, field, value)
    with pytest.raises(tahq.TahqError) as e:
        tahq.tahq_rotary_frequencies(cfg)
    assert e.value.status == 2
    assert _status("tahq_rotary_frequencies", tahq.make_rotary_config(1024), (C.c_uint64 * 512)()) == 3
    assert _status("tahq_rotary_frequencies", None, P) == 1 and _status("tahq_rotary_frequencies", cfg, None) == 1


@pytest.mark.parametrize("field, value, status", [
    ("tokens", 0, 2), ("tokens", 1 << 31, 2), ("q_heads", 0, 2), ("q_heads", 1 << 16, 2), ("k_heads", 65535, 2), ("head", 0, 2), ("head", 514, 3), ("rotated", 63, 2),
    ("rotated", 66, 2), ("layout", 2, 2), ("dtype", 2, 2), ("norm", 2, 2), ("accumulate", 2, 2), ("ldq", 255, 2), ("ldk", 127, 2), ("ldq_out", 255, 2),
    ("ldk_out", 127, 2), ("eps", 0.0, 2), ("eps", float("nan"), 2), ("magnitude", float("inf"), 2), ("struct_size", 8, 2)])
def test_heads_refuse_configurations(field, value, status):
    cfg = tahq.make_heads_config(10, 4, 2, 64, 64, tahq.BF16)
    setattr(cfg, field, value)
    assert _status("tahq_heads_forward", cfg, *[P] * 8, None) == status
    assert _status("tahq_heads_backward", cfg, *[P] * 13, BIG, None) == status and tahq.tahq_heads_workspace_size(cfg) == 0


def test_heads_refuse_arguments():
    cfg = tahq.make_heads_config(10, 4, 2, 64, 32, tahq.BF16)
    need = tahq.tahq_heads_workspace_size(cfg)
    good, back = [P] * 8, [P] * 13
    for i in range(8):
        assert _status("tahq_heads_forward", cfg, *good[:i], None, *good[i + 1:], None) == 1
    for i in range(13):
        assert _status("tahq_heads_backward", cfg, *back[:i], None, *back[i + 1:], BIG, None) == 1
    assert _status("tahq_heads_backward", cfg, *back, need - 1, None) == 5
    # elements' alignment for queries and keys, 8 bytes for positions, 16 for the others
    for i, step in ((0, 1), (1, 1), (2, 8), (3, 8), (4, 4), (5, 8), (6, 1), (7, 1)):
        assert _status("tahq_heads_forward", cfg, *good[:i], P + step, *good[i + 1:], None) == 6
    for i, step in ((0, 1), (2, 1), (4, 8), (6, 4), (8, 1), (10, 8), (12, 8)):
        assert _status("tahq_heads_backward", cfg, *back[:i], P + step, *back[i + 1:], BIG, None) == 6
    # what there is not is not given
    plain = tahq.make_heads_config(10, 4, 2, 64, 32, tahq.BF16, norm=0)
    assert _status("tahq_heads_forward", plain, *good, None) == 2 and tahq.tahq_heads_workspace_size(plain) == 0
    assert _status("tahq_heads_backward", plain, *back, BIG, None) == 2
    still = tahq.make_heads_config(10, 4, 2, 64, 0, tahq.BF16)
    assert _status("tahq_heads_forward", still, *good, None) == 2
    alone = tahq.make_heads_config(10, 4, 0, 64, 32, tahq.BF16)
    assert _status("tahq_heads_forward", alone, *good, None) == 2
    assert _status("tahq_heads_forward", None, *good, None) == 1 and _status("tahq_heads_backward", None, *back, BIG, None) == 1


def test_heads_differences():
    """The oracle's gradients against differences of its outputs: a step h leaves h^2 times a third derivative, of the size of 1, and 2^-53 / h."""
    g = np.random.default_rng(3)
    tokens, heads, head, rotated = 3, 2, 10, 6
    x, w, up = g.standard_normal((tokens, heads, head)), 1 + 0.2 * g.standard_normal(head), g.standard_normal((tokens, heads, head))
    positions, f = np.array([0, 5, -1000003]), heads64.frequencies(rotated)
    for pairs in (0, 1):
        run = lambda x, w: heads64.forward(x, w, positions, f, rotated, pairs, 1e-6, 1.25)[0]      # noqa: E731,B023
        dx, _, dw, _ = heads64.backward(up, x, w, positions, f, rotated, pairs, 1e-6, 1.25)
        h = 1e-5
        for at in ((0, 0, 0), (1, 1, 3), (2, 0, 9), (2, 1, 5)):
            step = np.zeros_like(x)
            step[at] = h
            assert abs(((run(x + step, w) - run(x - step, w)) * up).sum() / (2 * h) - dx[at]) < 1e-7
        for at in (0, 5, 9):
            step = np.zeros(head)
            step[at] = h
            assert abs(((run(x, w + step) - run(x, w - step)) * up).sum() / (2 * h) - dw[at]) < 1e-7


# ---------------------------------------------------------------- loss

@pytest.mark.parametrize("field, value, status", [("rows", 0, 2), ("rows", 1 << 31, 2), ("cols", 0, 2), ("cols", 65537, 3), ("rows", (1 << 23) + 1, 3), ("vocab", 0, 2), ("vocab", 1 << 31, 2), ("dtype", 2, 2),
                                                  ("weight_dtype", 2, 2), ("reduction", 3, 2), ("accumulate", 2, 2), ("struct_size", 8, 2)])
def test_loss_refuses_configurations(field, value, status):
    cfg = tahq.make_loss_config(10, 64, 100, tahq.BF16)
    setattr(cfg, field, value)
    assert tahq.tahq_loss_forward_workspace_size(cfg) == tahq.tahq_loss_backward_workspace_size(cfg) == 0
    assert _status("tahq_loss_forward", cfg, *[P] * 7, BIG, None) == status
    assert _status("tahq_loss_backward", cfg, *[P] * 8, BIG, None) == status


def test_loss_refuses_launches_of_2_to_the_32_lanes():
    for cfg in (tahq.make_loss_config((1 << 31) - 1, 8, (1 << 31) - 1, tahq.BF16), tahq.make_loss_config((1 << 31) - 1, 8, 100, tahq.F32)):
        assert tahq.tahq_loss_forward_workspace_size(cfg) == 0 and _status("tahq_loss_forward", cfg, *[P] * 7, BIG, None) == 3


def test_loss_refuses_arguments():
    cfg = tahq.make_loss_config(10, 64, 100, tahq.BF16)
    forward, backward = tahq.tahq_loss_forward_workspace_size(cfg), tahq.tahq_loss_backward_workspace_size(cfg)
    f = lambda *a: _status("tahq_loss_forward", cfg, *a, None)       # noqa: E731
    b = lambda *a: _status("tahq_loss_backward", cfg, *a, None)      # noqa: E731
    for i in range(7):
        assert f(*[P] * i, None, *[P] * (6 - i), forward) == 1
    assert f(*[P] * 7, forward - 1) == 5 and b(*[P] * 8, backward - 1) == 5
    for i in (0, 1, 2, 3, 7):
        assert b(*[P] * i, None, *[P] * (7 - i), backward) == 1
    assert b(P, P, P, P, P, None, None, P, backward) == 1
    for i, step in ((0, 8), (1, 4), (2, 4), (3, 8), (4, 8), (5, 8), (6, 8)):
        assert f(*[P] * i, P + step, *[P] * (6 - i), forward) == 6
    for i, step in ((0, 8), (1, 4), (2, 4), (3, 8), (4, 2), (5, 8), (6, 8), (7, 8)):
        assert b(*[P] * i, P + step, *[P] * (7 - i), backward) == 6
    with pytest.raises(ValueError):
        tahq.tahq_loss_forward(cfg, torch.zeros(10, 64), torch.zeros(100, 64), torch.zeros(10, dtype=torch.int64), None, None, None, None)
    with pytest.raises(ValueError):
        tahq.tahq_loss_forward(cfg, torch.zeros(10, 64, dtype=torch.bfloat16), torch.zeros(100, 64, dtype=torch.bfloat16), torch.zeros(10, dtype=torch.int32), None, None, None, None)


def test_loss_workspace_is_a_piece():
    """However large the vocabulary, the workspace holds a piece of it."""
    small, large = (tahq.make_loss_config(8192, 4096, vocab, tahq.BF16) for vocab in (50257, 1 << 22))
    for size in (tahq.tahq_loss_forward_workspace_size, tahq.tahq_loss_backward_workspace_size):
        assert size(large) <= size(small) + (300 << 20) < 2 << 30
    assert tahq.tahq_loss_backward_workspace_size(large) < 8192 * (1 << 22) // 8


def test_loss_differences():
    """The oracle's gradients against differences, as above."""
    g = torch.Generator().manual_seed(5)
    x, w = torch.randn(5, 4, generator=g, dtype=torch.float64), torch.randn(7, 4, generator=g, dtype=torch.float64)
    target, up = torch.tensor([3, -100, 0, 6, 2]), torch.rand(5, generator=g, dtype=torch.float64)
    run = lambda x, w: (loss64.forward(x, w, target, -100)[0] * up).sum()      # noqa: E731
    dx, dw, _ = loss64.backward(x, w, target, -100, up)
    h = 1e-5
    for at in ((0, 0), (1, 2), (4, 3)):
        step = torch.zeros_like(x)
        step[at] = h
        assert abs((run(x + step, w) - run(x - step, w)) / (2 * h) - dx[at]) < 1e-7
    for at in ((0, 0), (3, 2), (6, 3)):
        step = torch.zeros_like(w)
        step[at] = h
        assert abs((run(x, w + step) - run(x, w - step)) / (2 * h) - dw[at]) < 1e-7
