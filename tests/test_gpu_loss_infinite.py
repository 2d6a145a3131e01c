"""Infinite weights, masks of the lowest number and NaN, in every way that products go: the same whatever the number of tokens."""
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import loss64
from test_gpu_loss import HALF, IGNORE, KINDS, UNIT, _bounds, _make

pytestmark = pytest.mark.gpu

# fp32: up to 32 tokens straight from memory and through LDS, as such in small and middle tiles; in planes in middle and large tiles, with long rows, with rows that are copied.  bf16: each kind
SIZES = [(13, 33, 500, "f32"), (13, 64, 9001, "f32"), (70, 64, 300, "f32"), (200, 64, 16001, "f32"), (400, 64, 8300, "f32"), (161, 31, 17000, "f32"), (700, 64, 33003, "f32"),
         (1500, 1040, 33003, "f32"), (13, 33, 500, "bf16"), (70, 64, 300, "bf16"), (500, 96, 32601, "bf16")]


def _masked(vocab, run=True):
    """Two rows; with `run` also the last one and a run that fills some tiles and ends within one."""
    rows = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    rows[[0, 7]] = True
    if run:
        rows[vocab - 1] = True
        rows[vocab // 3:vocab // 3 + min(300, vocab // 4)] = True
    return rows


def _inputs(rows, cols, vocab, kind, run=True):
    x, weight, target, _ = _make(rows, cols, vocab, kind)
    x[:, 0] = 1                                          # a bias
    masked = _masked(vocab, run)
    free = (~masked).nonzero()[:, 0]
    target = torch.where((target != IGNORE) & masked[target.clamp_min(0)], free[target % len(free)], target)
    return x, weight, target, masked


def _run(x, weight, target, kind):
    loss = tahq.LinearLoss(tahq.make_loss_config(*x.shape, len(weight), KINDS[kind][0], reduction=tahq.LOSS_SUM))
    loss.forward(x, weight, target)
    loss.backward(x, weight, target)
    return loss


def _check(loss, x, weight, target, masked, kind, channels):
    """As if the masked rows were not there; the bounds of test_gpu_loss.py."""
    vocab = len(weight)
    rest, place = weight[~masked], torch.cumsum((~masked).long(), 0) - 1
    fewer = torch.where(target == IGNORE, target, place[target.clamp(0, vocab - 1)])
    want, want_lse = loss64.forward(x, rest, fewer, IGNORE)
    off, lse_off, p_off = _bounds(x, rest, fewer, kind)
    assert ((loss.losses.double() - want).abs() <= off + lse_off + UNIT * want.abs()).all() and ((loss.lse.double() - want_lse).abs() <= lse_off).all()
    counts = target != IGNORE
    want_x, want_w, d = loss64.backward(x, rest, fewer, IGNORE, torch.ones(len(x), dtype=torch.float64, device="cuda"))
    p = d.abs()
    at = torch.arange(len(x), device="cuda")[counts]
    p[at, fewer[counts]] = (d[at, fewer[counts]] + 1).abs()
    each = torch.where(counts[:, None], p * p_off[:, None] + (HALF[kind] + 4 * UNIT) * d.abs() + 2 * UNIT * p, torch.zeros_like(p))
    w_abs, x_abs = rest.double().abs(), x.double().abs()
    bound = each @ w_abs + (2 * vocab + 16) * UNIT * (d.abs() @ w_abs) + HALF[kind] * want_x.abs() + 1e-38
    assert ((loss.grad_x.double() - want_x).abs() <= bound)[:, channels].all()
    bound = each.t().contiguous() @ x_abs + (2 * len(x) + 16) * UNIT * (d.abs().t().contiguous() @ x_abs) + HALF[kind] * want_w.abs() + 1e-38
    assert ((loss.grad_weight[~masked].double() - want_w).abs() <= bound).all() and (loss.grad_weight[masked] == 0).all()


@pytest.mark.parametrize("rows, cols, vocab, kind", SIZES)
def test_bias_of_minus_infinity(rows, cols, vocab, kind):
    """Probability 0, and a gradient of 0 times infinity in the bias' channel alone."""
    x, weight, target, masked = _inputs(rows, cols, vocab, kind)
    weight[masked, 0] = float("-inf")
    loss = _run(x, weight, target, kind)
    _check(loss, x, weight, target, masked, kind, slice(1, None))
    assert loss.grad_x[target != IGNORE, 0].isnan().all() and (loss.grad_x[target == IGNORE] == 0).all()


@pytest.mark.parametrize("rows, cols, vocab, kind", SIZES)
def test_bias_of_the_lowest_number(rows, cols, vocab, kind):
    x, weight, target, masked = _inputs(rows, cols, vocab, kind, False)
    weight[masked, 0] = torch.finfo(weight.dtype).min
    _check(_run(x, weight, target, kind), x, weight, target, masked, kind, slice(None))


@pytest.mark.parametrize("rows, cols, vocab, kind", SIZES)
@pytest.mark.parametrize("value", (None, -1e38, -1e30, -1e12, -1e5))
def test_runs_of_large_negative_biases(rows, cols, vocab, kind, value):
    """Masks (None: the lowest number) that leave nothing else in some tiles."""
    x, weight, target, masked = _inputs(rows, cols, vocab, kind)
    weight[masked, 0] = torch.finfo(weight.dtype).min if value is None else value
    _check(_run(x, weight, target, kind), x, weight, target, masked, kind, slice(None))


@pytest.mark.parametrize("rows, cols, vocab, kind", SIZES)
def test_rows_of_minus_infinity(rows, cols, vocab, kind):
    """Of positive hidden states: logits of -infinity, losses of targets among them infinity."""
    x, weight, target, masked = _inputs(rows, cols, vocab, kind)
    x = x.abs() + 0.5
    weight[masked] = float("-inf")
    loss = _run(x, weight, target, kind)
    want, want_lse = loss64.forward(x, weight, target, IGNORE)
    off, lse_off, _ = _bounds(x, weight[~masked], target, kind)
    assert ((loss.losses.double() - want).abs() <= off + lse_off + UNIT * want.abs()).all() and ((loss.lse.double() - want_lse).abs() <= lse_off).all()
    assert loss.grad_weight.isfinite().all() and (loss.grad_weight[masked] == 0).all()
    there = target != IGNORE
    first = int(there.nonzero()[0])
    target[first] = 7
    loss.forward(x, weight, target)
    assert loss.losses[first] == float("inf") and loss.losses[first + 1:].isfinite().all() and loss.lse.isfinite().all()


@pytest.mark.parametrize("rows, cols, vocab, kind", SIZES)
@pytest.mark.parametrize("value", (float("nan"), float("inf")))
def test_a_token_that_is_none(rows, cols, vocab, kind, value):
    """NaN or infinity in a hidden state stays in its token, forward and in its gradient; the weight's gradient has it."""
    x, weight, target, _ = _inputs(rows, cols, vocab, kind)
    clean = _run(x, weight, target, kind)
    bad = int((target != IGNORE).nonzero()[-1])
    x[bad, cols // 2] = value
    loss = _run(x, weight, target, kind)
    others = torch.arange(rows, device="cuda") != bad
    assert not loss.losses[bad].isfinite() and loss.grad_x[bad].isnan().all() and loss.grad_weight.isnan().any()
    off, lse_off, p_off = _bounds(torch.where(others[:, None], x, torch.zeros_like(x)), weight, target, kind)
    # as such instead of in planes where a tile has a NaN: either is as near to 64 bits as the bounds say
    assert ((loss.losses - clean.losses).double().abs() <= 2 * (off + lse_off) + 2 * UNIT * clean.losses.double().abs())[others].all()
    assert loss.grad_x[others].isfinite().all()


@pytest.mark.parametrize("rows, cols, vocab, kind", SIZES)
@pytest.mark.parametrize("size", (1e5, 1e8, 1e30))
def test_large_logits(rows, cols, vocab, kind, size):
    """Every token's largest logits are two equal ones of `size` and far above the others, and the target is one of the two: a loss of log 2, off by lse's
    rounding; p is 1 / 2 twice, off by that of lse, or 1 where that is all of it."""
    x, weight, target, _ = _inputs(rows, cols, vocab, kind, False)
    weight[:, 0] = 0
    counts = target != IGNORE
    x[:, 0] = 1
    x[:, 1:] = 0
    weight[[3, vocab - 2], 0] = size
    size = float(weight[3, 0])
    target = torch.where(counts, torch.where(torch.arange(rows, device="cuda") % 2 == 0, 3, vocab - 2), target)
    loss = _run(x, weight, target, kind)
    ulp = 2.0 ** -23 * size
    assert ((loss.lse[counts].double() - size).abs() <= ulp + 1).all() and ((loss.losses[counts].double()).abs() <= ulp + 1).all()
    assert loss.grad_x.isfinite().all() and loss.grad_weight.isfinite().all()
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    rest[[3, vocab - 2]] = False
    assert (loss.grad_weight[rest] == 0).all()


@pytest.mark.parametrize("reduction", (tahq.LOSS_NONE, tahq.LOSS_SUM, tahq.LOSS_MEAN))
@pytest.mark.parametrize("value", (float("nan"), float("inf")))
@pytest.mark.parametrize("accumulate", (0, 1))
def test_no_token_adds_nothing(reduction, value, accumulate):
    """Gradients without a token that counts are 0, or what was there, whatever the loss came back with: 0 / 0 of a mean, say."""
    x, weight, target, _ = _make(40, 64, 300, "bf16", 1.1)
    loss = tahq.LinearLoss(tahq.make_loss_config(40, 64, 300, tahq.BF16, reduction=reduction, accumulate=accumulate))
    loss.forward(x, weight, target)
    if accumulate:
        loss.grad_weight.fill_(3.0)
    grad_x, grad_w = loss.backward(x, weight, target, torch.full((40 if reduction == tahq.LOSS_NONE else 1,), value, device="cuda"))
    assert (grad_x == 0).all() and (grad_w == (3 if accumulate else 0)).all()
