"""Inputs of losses over a vocabulary that show what single products of fp32 and their long sums lose (csrc/tahq_loss_tiles.hpp), how much that may be, and
the products in planes of bf16 worked out on the CPU."""
import torch

UNIT = 2.0 ** -24           # half a unit in the last place of an fp32 number
AMPLITUDE, LOW = 64.0, 2.0 ** -10

# A logit or a gradient that is one product of two fp32 numbers.  In planes: the products that are left out are 2^-24 of it together, and six products
# go one after another into one sum, each off by a rounding of it, two where the matrix instruction drops what lies below its largest addend's last place.
ONE_PRODUCT = 14 * UNIT
# p, next to 1: lse of a single logit that counts, the difference, its product with log2(e), the power of two, and the factor
PROBABILITY = 16 * UNIT


def single_products(rows, cols, vocab, device="cpu", seed=1):
    """(x, weight, target, factor, winner): token n has one channel of its own that is not 0, of magnitude 64 to 128; there the weight's row `winner[n]` makes a logit of 0.06
    to 0.12, and all others at most -32, so that p is 1 for the winner.  Numbers have all 24 bits."""
    assert rows <= cols and rows < vocab
    g = torch.Generator(device=device).manual_seed(seed)
    some = lambda *s: (1 + torch.rand(*s, generator=g, device=device, dtype=torch.float64)).float()      # noqa: E731
    x = torch.zeros(rows, cols, device=device)
    n = torch.arange(rows, device=device)
    x[n, n] = AMPLITUDE * some(rows)
    weight = -0.5 * some(vocab, cols)
    order = torch.randperm(vocab, generator=g, device=device)
    winner = order[:rows]
    weight[winner, n] = LOW * some(rows)
    target = order[torch.randint(rows, vocab, (rows,), generator=g, device=device)] if vocab > 2 * rows else order[(n + 1) % rows]
    return x, weight, target, some(rows), winner


def wanted(x, weight, target, factor, winner):
    """Of single_products in 64 bits: logits of target and winner, the hidden states' gradient and the magnitude of its terms; and the weight's gradient at the winners' and the
    targets' rows in the tokens' own channels."""
    n = torch.arange(x.shape[0], device=x.device)
    a, g = x[n, n].double(), factor.double()
    won, lost = weight[winner].double(), weight[target].double()
    return {"target": a * lost[n, n], "winner": a * won[n, n], "grad_x": g[:, None] * (won - lost), "grad_x_size": g[:, None] * (won.abs() + lost.abs()), "grad_w": g * a}


def split(x):
    """Three bf16 whose sum an fp32 number is, each what is left rounded to nearest."""
    planes, left = [], x.clone()
    for _ in range(3):
        p = left.bfloat16().float()
        planes.append(p.double())
        left = left - p
    return planes


def product(x, y, products=6):
    """x y as sums of so many products of planes, largest first, without the sums' roundings."""
    a, b = split(x), split(y)
    order = [(0, 0), (0, 1), (1, 0), (0, 2), (2, 0), (1, 1)]
    return sum(a[i] * b[j] for i, j in order[:products])


def long_sum(instructions, parts, half=0.5):
    """Standard deviation of a sum's error, over the sum's own: `parts` sums of so many instructions' results one after another, which are then added up.  Every instruction's result
    is off by two roundings of what has been added so far at most, as if drawn from all of that, which has `half` of the whole sum's square on
    average."""
    return 2 * UNIT * ((instructions * half / 3) ** 0.5 + (parts * half / 3) ** 0.5)
