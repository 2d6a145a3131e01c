"""What fp32 losses and gradients lose in single products and in long sums: bounds that fewer products of planes, or one chain of sums, do not keep (test_loss_products_host.py)."""
import pytest
import torch

import loss_products as lp
import paper_2506_01352_amd as tahq

pytestmark = pytest.mark.gpu

UNIT = lp.UNIT


def _run(x, weight, target, factor=None, reduction=tahq.LOSS_NONE):
    cfg = tahq.make_loss_config(*x.shape, weight.shape[0], tahq.F32, reduction=reduction)
    loss = tahq.LinearLoss(cfg)
    loss.forward(x, weight, target)
    loss.backward(x, weight, target, factor)
    return loss


# fp32 as such: small, middle tiles, up to 32 tokens; in planes: middle tiles, large ones (one run of a gradient's sums, several), rows that are copied
@pytest.mark.parametrize("rows, cols, vocab", [(20, 32, 500), (20, 33, 9001), (66, 272, 4099), (200, 208, 16001), (400, 416, 8300), (161, 161, 17000), (700, 704, 33003), (1100, 1104, 33003)])
def test_single_products(rows, cols, vocab):
    """A logit is lse - loss, off by the loss's rounding: |loss| and |lse| are below 256, a loss's rounding is one of it.  Gradients are sums of two
    products of unlike rows, rounded; what the other rows add is below 2^-40 of them."""
    x, weight, target, factor, winner = lp.single_products(rows, cols, vocab, "cuda")
    want = lp.wanted(x, weight, target, factor, winner)
    loss = _run(x, weight, target, factor)
    got = loss.lse.double() - loss.losses.double()
    assert ((got - want["target"]).abs() <= lp.ONE_PRODUCT * want["target"].abs() + UNIT * loss.losses.double().abs()).all()
    assert ((loss.lse.double() - want["winner"]).abs() <= lp.ONE_PRODUCT * want["winner"] + 16 * UNIT).all()
    off = lp.ONE_PRODUCT + lp.PROBABILITY + 2 * UNIT
    assert ((loss.grad_x.double() - want["grad_x"]).abs() <= off * want["grad_x_size"]).all()
    n = torch.arange(rows, device="cuda")
    assert ((loss.grad_weight[winner, n].double() - want["grad_w"]).abs() <= off * want["grad_w"]).all()
    assert ((loss.grad_weight[target, n].double() + want["grad_w"]).abs() <= off * want["grad_w"]).all()


def _normal(rows, cols, vocab, size):
    g = torch.Generator(device="cuda").manual_seed(7)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    return size * make(rows, cols), make(vocab, cols) * cols ** -0.5, torch.randint(0, vocab, (rows,), generator=g, device="cuda")


@pytest.mark.parametrize("rows, cols, vocab, instructions", [
    (1024, 65536, 4100, 192),                            # planes, middle tiles, which the plan takes for long rows
    (400, 1024, 33003, 384), (1500, 1024, 33003, 384),   # planes, middle and large tiles, one part
    (200, 16384, 16001, 384), (200, 1600, 50257, 384),   # as such, middle tiles
    (66, 16384, 4099, 384)])                             # as such, small ones
def test_long_rows(rows, cols, vocab, instructions):
    """Logits of standard deviation 8 as lse - loss: a sum in parts, and the loss's rounding, at most 2^-24 of it; loss and lse have less than 8 such logits."""
    size = 8.0
    x, weight, target = _normal(rows, cols, vocab, size)
    loss = tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, tahq.F32, reduction=tahq.LOSS_NONE), training=False)
    loss.forward(x, weight, target)
    want = (x.double() * weight[target].double()).sum(1)
    off = (loss.lse.double() - loss.losses.double() - want).square().mean().sqrt()
    planes = rows >= 384
    each = 16 / 6 if planes else 2                       # columns of an instruction
    parts = max(cols / each / instructions, 1)
    bound = size * (lp.long_sum(min(instructions, cols / each), parts) + 8 * UNIT / 3 ** 0.5)
    assert float(off) <= bound, (float(off), bound)


@pytest.mark.parametrize("rows, cols, vocab", [(4100, 2056, 20000), (16400, 5120, 8192), (16400, 64, 4099), (300, 4104, 4200)])
def test_long_sums_of_gradients(rows, cols, vocab):
    """Gradients of logits next to 0: of a hidden state it is its target's row nearly alone, from a random place of the sum on; of the weight, of some tokens at random places.  Of
    a sum's square half is there on average; parts hold 384 instructions at the most.  p is off by lse's rounding, up to 16 UNIT as lse is 8 to 16, and 16 more."""
    x, weight, target = _normal(rows, cols, vocab, 2.0 ** -10)
    loss = _run(x, weight, target, reduction=tahq.LOSS_SUM)
    d = torch.softmax(x.double() @ weight.double().t(), 1)
    d[torch.arange(rows, device="cuda"), target] -= 1
    for got, want, terms in ((loss.grad_x, d @ weight.double(), vocab), (loss.grad_weight, d.t().contiguous() @ x.double(), rows)):
        instructions = terms / 16 * 6
        bound = lp.long_sum(min(instructions, 384), max(instructions / 384, 1)) + 32 * UNIT / vocab ** 0.5 + 2 * UNIT
        off = float((got.double() - want).norm() / want.norm())
        assert off <= bound, (off, bound)


@pytest.mark.parametrize("reduction", (tahq.LOSS_NONE, tahq.LOSS_SUM))
@pytest.mark.parametrize("accumulate, wide", [(1, tahq.F32), (1, tahq.BF16), (0, tahq.BF16)])
def test_runs_that_are_added_to_a_gradient(reduction, accumulate, wide):
    """More tokens than one run of a large tile's sums: added to what is there once, in fp32, and rounded once where the gradient is bf16."""
    rows, cols, vocab = 1100, 1104, 33003
    x, weight, target, factor, winner = lp.single_products(rows, cols, vocab, "cuda")
    if reduction == tahq.LOSS_SUM:
        factor = factor[:1]
    want = lp.wanted(x, weight, target, factor.expand(rows), winner)
    cfg = tahq.make_loss_config(rows, cols, vocab, tahq.F32, wide, reduction, accumulate=accumulate)
    loss = tahq.LinearLoss(cfg)
    loss.forward(x, weight, target)
    before = 3.0 if accumulate else 0.0
    loss.grad_weight.fill_(before)
    grad = loss.backward(x, weight, target, factor)[1].double()
    half = 2.0 ** -8 if wide == tahq.BF16 else UNIT
    n = torch.arange(rows, device="cuda")
    for at, value in ((winner, want["grad_w"]), (target, -want["grad_w"])):
        off = (lp.ONE_PRODUCT + lp.PROBABILITY + 4 * UNIT) * value.abs() + half * (value + before).abs() + 2 * UNIT * before
        assert ((grad[at, n] - (value + before)).abs() <= off).all()
    untouched = torch.ones_like(grad, dtype=torch.bool)
    untouched[winner, n] = untouched[target, n] = False
    assert (grad[untouched] - before).abs().max() <= 1e-9
