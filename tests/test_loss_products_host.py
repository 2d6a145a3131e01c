"""Products of fp32 as products of planes of bf16, on the CPU: what they lose, and that the bounds of the GPU tests tell six products from five or three."""
from fractions import Fraction

import pytest
import torch

import loss_products as lp


def test_what_six_products_leave_out():
    """x2 y3 + x3 y2 + x3 y3: |x2| reaches 2^-8 |x| and |x3| 2^-17 |x|, so 2^-24 of |x y| together, for numbers next to 1 that round the wrong way twice."""
    worst = torch.tensor([float.fromhex("0x1.00ff8p+0")])
    exact = Fraction(float(worst)) ** 2
    assert [float(p) for p in lp.split(worst)] == [1.0, 2.0 ** -8, -(2.0 ** -17)]
    left = abs(Fraction(float(lp.product(worst, worst))) - exact) / exact
    assert Fraction(19, 10) * Fraction(1, 1 << 25) < left <= Fraction(1, 1 << 24)
    g = torch.Generator().manual_seed(2)
    x, y = ((1 + torch.rand(1 << 20, generator=g, dtype=torch.float64)).float() for _ in range(2))
    assert ((lp.product(x, y) - x.double() * y.double()).abs() <= 2.0 ** -24 * x.double() * y.double()).all()
    assert (sum(lp.split(x)) == x.double()).all()


@pytest.mark.parametrize("products, good", [(6, True), (5, False), (3, False), (1, False)])
def test_single_products_tell_them_apart(products, good):
    x, weight, target, factor, winner = lp.single_products(161, 161, 17000)
    want = lp.wanted(x, weight, target, factor, winner)
    n = torch.arange(161)
    a = x[n, n]
    off = (lp.product(a, weight[target, n], products) - want["target"]).abs()
    assert (off <= lp.ONE_PRODUCT * want["target"].abs()).all() == good
    off = (lp.product(factor[:, None], weight[winner], products) - lp.product(factor[:, None], weight[target], products) - want["grad_x"]).abs()
    assert (off <= (lp.ONE_PRODUCT + lp.PROBABILITY) * want["grad_x_size"]).all() == good
    off = (lp.product(factor, a, products) - want["grad_w"]).abs()
    assert (off <= (lp.ONE_PRODUCT + lp.PROBABILITY) * want["grad_w"]).all() == good


def test_winners_win():
    x, weight, target, _, winner = lp.single_products(161, 161, 17000)
    p = torch.softmax(x.double() @ weight.double().t(), 1)
    n = torch.arange(161)
    assert (winner != target).all() and (1 - p[n, winner] < 17000 * 1.3e-14).all()


@pytest.mark.parametrize("columns", (32768, 65536))
def test_long_sums_tell_parts_apart(columns):
    """Sums of fp32 products with a rounding after every sixteen columns' six products each, in one chain and in parts of 512 columns."""
    g = torch.Generator().manual_seed(3)
    x, y = (torch.randn(256, columns, generator=g) for _ in range(2))
    y *= columns ** -0.5
    steps = torch.cat([(a.view(256, -1, 16) * b.view(256, -1, 16)).sum(2)[:, :, None] for a, b in
                       ((lp.split(x)[i], lp.split(y)[j]) for i, j in ((0, 0), (0, 1), (0, 2), (1, 0), (1, 1), (2, 0)))], 2).flatten(1).float()
    want = steps.double().sum(1)

    def chain(v):
        s = torch.zeros(len(v))
        for k in range(v.shape[1]):
            s = s + v[:, k]
        return s

    parts = columns // 512
    bound = lp.long_sum(192, parts)
    rms = lambda s: float((s.double() - want).square().mean().sqrt())      # noqa: E731
    assert rms(chain(torch.stack([chain(p) for p in steps.chunk(parts, 1)], 1))) <= bound < rms(chain(steps))
