"""The loss over a vocabulary through the C ABI against its 64-bit definition, forward and backward."""
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import loss64

pytestmark = pytest.mark.gpu

KINDS = {"f32": (tahq.F32, torch.float32), "bf16": (tahq.BF16, torch.bfloat16)}
UNIT = 2.0 ** -24           # half a unit in the last place of an fp32 number
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
IGNORE = -100


def _make(rows, cols, vocab, kind, ignored=0.25, seed=1, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    make = lambda *s: torch.randn(*s, generator=g, device=device)      # noqa: E731
    weight = make(vocab, cols) * cols ** -0.5
    target = torch.randint(0, vocab, (rows,), generator=g, device=device)
    x = make(rows, cols) + 6 * torch.rand(rows, 1, generator=g, device=device) * weight[target]
    target[torch.rand(rows, generator=g, device=device) < ignored] = IGNORE
    return x.to(KINDS[kind][1]), weight.to(KINDS[kind][1]), target, torch.rand(rows, generator=g, device=device)


def _bounds(x, weight, target, kind):
    """How far a logit may be off, and lse, per token; and the relative error of a probability.

    A logit is a sum of `cols` products in fp32, each addition off by a rounding of what has been added so far, two where the matrix instruction drops
    what lies below its largest addend's last place.  exp(l - top): the difference is rounded, times log2(e) rounded again, so the exponent is off by 3 UNIT |l -
    top|, and the hardware's power of two by 2 UNIT; sums of 64 values in a row, a tree over parts, rounding of the logarithm: 160 UNIT."""
    size = x.double().abs() @ weight.double().abs().t()
    off = (2 * x.shape[1] + 2) * UNIT * size.amax(1)
    logits = x.double() @ weight.double().t()
    top = logits.amax(1)
    reach = ((top[:, None] - logits) * torch.softmax(logits, 1)).sum(1)
    parts = -(-weight.shape[0] // 32)
    lse_off = off + UNIT * (160 + 3 * reach + parts + 4 * torch.logsumexp(logits, 1).abs() + 2 * top.abs())
    spread = (logits.amax(1) - logits.amin(1))
    return off, lse_off, off + lse_off + UNIT * (3 * (spread + 2) + 4 + 2 * torch.logsumexp(logits, 1).abs())


def _check(rows, cols, vocab, kind, reduction=tahq.LOSS_MEAN, ignored=0.25, weight_dtype=None, grad=True, seed=1, x_wanted=True, w_wanted=True, accumulate=0):
    x, weight, target, up = _make(rows, cols, vocab, kind, ignored, seed)
    cfg = tahq.make_loss_config(rows, cols, vocab, KINDS[kind][0], weight_dtype, reduction, IGNORE, accumulate)
    need = tahq.tahq_loss_forward_workspace_size(cfg)
    workspace = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    losses, lse, total = (torch.full((n + 4,), 7.0, device="cuda") for n in (rows, rows, 2))
    tahq.tahq_loss_forward(cfg, x, weight, target, losses, lse, total, workspace[:need])
    torch.cuda.synchronize()
    assert (workspace[need:] == 0xFF).all() and all((t[n:] == 7).all() for t, n in ((losses, rows), (lse, rows), (total, 2)))
    want, want_lse = loss64.forward(x, weight, target, IGNORE)
    off, lse_off, p_off = _bounds(x, weight, target, kind)
    loss_off = off + lse_off + UNIT * want.abs()
    assert ((losses[:rows].double() - want).abs() <= loss_off).all() and ((lse[:rows].double() - want_lse).abs() <= lse_off).all()
    counts = target != IGNORE
    assert (losses[:rows][~counts] == 0).all() and (lse[:rows][~counts] == 0).all()
    reduced, n = loss64.reduced(want, target, IGNORE, reduction)
    sum_off = (loss_off * counts).sum() / (max(n, 1) if reduction == tahq.LOSS_MEAN else 1)
    assert total[1] == n and abs(total[0].double() - reduced) <= sum_off + (rows / 512 + 16) * UNIT * want.abs().sum() / (max(n, 1) if reduction == tahq.LOSS_MEAN else 1)
    if not grad:
        return
    need = tahq.tahq_loss_backward_workspace_size(cfg)
    workspace = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    wide = KINDS["bf16" if cfg.weight_dtype == tahq.BF16 else "f32"][1]
    grad_x = torch.full((rows + 1, cols), 7.0, dtype=x.dtype, device="cuda")
    grad_w = torch.full((vocab + 1, cols), 7.0, dtype=wide, device="cuda")
    grad_loss = up if reduction == tahq.LOSS_NONE else up[:1]
    tahq.tahq_loss_backward(cfg, x, weight, target, lse, grad_loss, grad_x if x_wanted else None, grad_w if w_wanted else None, workspace[:need])
    torch.cuda.synchronize()
    assert (workspace[need:] == 0xFF).all() and (grad_x[rows:] == 7).all() and (grad_w[vocab:] == 7).all()
    g = (up if reduction == tahq.LOSS_NONE else up[:1].expand(rows)).double() / (max(n, 1) if reduction == tahq.LOSS_MEAN else 1)
    want_x, want_w, d = loss64.backward(x, weight, target, IGNORE, g)
    # every p - [v = t] is off by p's error and its rounding for the matrix cores (with LOSS_NONE after the product with g); then sums in fp32
    counted = (counts * g.abs())[:, None]
    p = d.abs().clone()
    at = torch.arange(rows, device="cuda")[counts]
    p[at, target[counts]] = (d[at, target[counts]] + g[counts]).abs()
    each = p * p_off[:, None] + (HALF[kind] + 4 * UNIT) * d.abs() + 2 * UNIT * p
    each = torch.where(counted > 0, each, torch.zeros_like(each))
    w_abs, x_abs = weight.double().abs(), torch.where(counts[:, None], x.double().abs(), torch.zeros(()).double().cuda())
    if x_wanted:
        bound = each @ w_abs + (2 * vocab + 16) * UNIT * (d.abs() @ w_abs) + HALF[kind] * want_x.abs() + 1e-38
        assert ((grad_x[:rows].double() - want_x).abs() <= bound).all() and (grad_x[:rows][~counts] == 0).all()
    else:
        assert (grad_x == 7).all()
    if w_wanted:
        before = 7.0 if accumulate else 0.0
        out_half = HALF["bf16" if cfg.weight_dtype == tahq.BF16 else "f32"]
        bound = each.t().contiguous() @ x_abs + (2 * rows + 16) * UNIT * (d.abs().t().contiguous() @ x_abs) + out_half * (want_w + before).abs() + UNIT * before + 1e-38
        assert ((grad_w[:vocab].double() - (want_w + before)).abs() <= bound).all()
    else:
        assert (grad_w == 7).all()


SMALL = [(1, 1, 1), (1, 8, 2), (2, 7, 3), (5, 32, 127), (31, 33, 128), (32, 40, 129), (33, 96, 500), (64, 257, 1000), (130, 1600, 257), (300, 64, 5003), (129, 1001, 999)]


@pytest.mark.parametrize("rows, cols, vocab", SMALL)
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("reduction", (tahq.LOSS_NONE, tahq.LOSS_SUM, tahq.LOSS_MEAN))
def test_small(rows, cols, vocab, kind, reduction):
    _check(rows, cols, vocab, kind, reduction, weight_dtype=tahq.F32 if reduction == tahq.LOSS_SUM else None)


# what takes the largest tiles: of logits, of the hidden states' gradient, of the weight's, with rows of whole stages (an odd number of them) and without;
# several pieces of the vocabulary backward, with the last one ragged; shared sums over the vocabulary; more tokens than one workgroup counts
LARGE = [(300, 40, 33003), (4100, 4100, 70), (40, 4104, 4200), (4100, 40, 40001), (257, 512, 9000), (9000, 24, 300), (1030, 2056, 4099), (300, 96, 33003), (1030, 2080, 4099),
         (4100, 64, 40001), (40, 4128, 4201), (500, 40, 32601), (500, 96, 32601)]


@pytest.mark.parametrize("rows, cols, vocab", LARGE)
def test_large(rows, cols, vocab):
    _check(rows, cols, vocab, "bf16")


# fp32 as three planes of bf16, in every kind of tile: of logits, of both gradients; in one direction alone; several pieces of the vocabulary
@pytest.mark.parametrize("rows, cols, vocab", [(1030, 260, 4099), (4100, 30, 17001), (700, 64, 33003), (1030, 2056, 4099), (300, 4104, 4200), (230, 48, 777), (640, 33, 500),
                                               (161, 31, 300), (6200, 16, 30001), (200, 64, 16001), (100, 33, 32001), (66, 260, 4099), (300, 64, 11003), (161, 31, 17000)])
def test_large_f32(rows, cols, vocab):
    _check(rows, cols, vocab, "f32")


# up to 32 tokens: runs of 256 bytes of a row, an even and an odd number of them, and what is left, with one wavefront to the channels and with eight;
# several pieces of the vocabulary; through LDS
@pytest.mark.parametrize("rows, cols, vocab", [(7, 1001, 700), (32, 1600, 999), (3, 4099, 515), (20, 384, 300), (9, 256, 33), (32, 127, 64), (1, 64, 31), (17, 130, 65), (2, 8, (1 << 22) + 700), (5, 1001, 9001), (32, 259, 8193), (20, 384, 9001), (3, 1600, 8200),
                                               (5, 4097, 100), (31, 2048, 640)])
@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_few(rows, cols, vocab, kind):
    _check(rows, cols, vocab, kind, ignored=0.3)


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("cols", (31, 256, 1600))
def test_few_tokens_that_do_not_count_and_targets_that_are_none(kind, cols):
    x, weight, target, _ = _make(13, cols, 301, kind, 0.0)
    target[::3] = IGNORE
    target[1], target[4] = 301, -7
    clean = tahq.LinearLoss(tahq.make_loss_config(13, cols, 301, KINDS[kind][0], reduction=tahq.LOSS_SUM), training=False)
    clean.forward(x, weight, target)
    losses, lse = clean.losses.clone(), clean.lse.clone()
    x[::3] = float("nan")
    clean.forward(x, weight, target)
    bad = torch.zeros(13, dtype=torch.bool, device="cuda")
    bad[1] = bad[4] = True
    assert torch.equal(clean.lse, lse) and lse.isfinite().all() and (lse[::3] == 0).all() and (losses[::3] == 0).all()
    assert clean.losses[bad].isnan().all() and torch.equal(clean.losses[~bad], losses[~bad]) and clean.total[1] == 8 and clean.total[0].isnan()
    want, want_lse = loss64.forward(x[~bad], weight, target[~bad], IGNORE)
    off, lse_off, _ = _bounds(torch.nan_to_num(x[~bad]), weight, target[~bad], kind)
    assert ((losses[~bad].double() - want).abs() <= off + lse_off + UNIT * want.abs()).all() and ((lse[~bad].double() - want_lse).abs() <= lse_off).all()


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("ignored", (0.0, 1.1))
def test_all_or_none_count(kind, ignored):
    for reduction in (tahq.LOSS_NONE, tahq.LOSS_SUM, tahq.LOSS_MEAN):
        _check(70, 72, 300, kind, reduction, ignored)


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("wide", (tahq.F32, tahq.BF16))
def test_weight_gradient_is_added_to(kind, wide):
    _check(70, 72, 300, kind, weight_dtype=wide, accumulate=1)


@pytest.mark.parametrize("x_wanted, w_wanted", [(True, False), (False, True)])
def test_one_gradient_alone(x_wanted, w_wanted):
    _check(70, 72, 300, "bf16", x_wanted=x_wanted, w_wanted=w_wanted)


def test_shares_of_several_pieces():
    """Few tiles whose sums over the vocabulary are shared by many workgroups, over two pieces of it of unlike length."""
    _check(544, 33, 246528 + 65600, "bf16")


def test_statistics_of_several_pieces():
    """More tokens times vocabulary than a piece of statistics holds; the definition a thousand tokens at a time."""
    rows, cols, vocab = 65536, 8, 70001
    x, weight, target, _ = _make(rows, cols, vocab, "bf16", 0.0)
    cfg = tahq.make_loss_config(rows, cols, vocab, tahq.BF16)
    loss = tahq.LinearLoss(cfg, training=False)
    loss.forward(x, weight, target)
    for first in range(0, rows, 8192):
        part = slice(first, first + 1024)
        want, want_lse = loss64.forward(x[part], weight, target[part], IGNORE)
        off, lse_off, _ = _bounds(x[part], weight, target[part], "bf16")
        assert ((loss.losses[part].double() - want).abs() <= off + lse_off + UNIT * want.abs()).all() and ((loss.lse[part].double() - want_lse).abs() <= lse_off).all()


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("cols", (64, 33))
def test_ignored_tokens_may_hold_anything(kind, cols):
    """NaN and infinities in hidden states of tokens that do not count change nothing, whatever the other tokens' places."""
    rows, vocab = 150, 300
    x, weight, target, _ = _make(rows, cols, vocab, kind)
    x = torch.where((target == IGNORE)[:, None], torch.zeros_like(x), x)
    dirty = x.clone()
    dirty[target == IGNORE] = float("nan")
    dirty[(target == IGNORE).nonzero()[::2, 0]] = float("inf")
    loss = tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, KINDS[kind][0]))
    got = []
    for v in (x, dirty):
        total = loss.forward(v, weight, target).clone()
        got.append((total, loss.losses.clone(), loss.lse.clone(), *(t.clone() for t in loss.backward(v, weight, target))))
    assert all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(*got))


def test_targets_that_are_none():
    """A target outside the vocabulary: NaN in the token's loss, its gradient and the weight's; the others' losses stay."""
    x, weight, target, _ = _make(40, 64, 300, "bf16", 0.0)
    loss = tahq.LinearLoss(tahq.make_loss_config(40, 64, 300, tahq.BF16, reduction=tahq.LOSS_SUM))
    loss.forward(x, weight, target)
    good = loss.losses.clone()
    bad = target.clone()
    bad[3], bad[17], bad[30] = 300, -1, 1 << 40
    total = loss.forward(x, weight, bad)
    wrong = torch.zeros(40, dtype=torch.bool, device="cuda")
    wrong[[3, 17, 30]] = True
    assert total.isnan().all() and loss.losses[wrong].isnan().all() and torch.equal(loss.losses[~wrong], good[~wrong]) and loss.total[1] == 40
    grad_x, grad_w = loss.backward(x, weight, bad)
    assert grad_x[wrong].isnan().all() and grad_x[~wrong].isfinite().all() and grad_w.isnan().all()


@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_infinite_and_large_logits(kind):
    """A weight row of -infinity gives probability 0; logits of thousands do not overflow; a NaN in a hidden state stays in its token."""
    x, weight, target, _ = _make(40, 64, 300, kind, 0.0)
    big = (x.float() * 300).to(x.dtype)
    loss = tahq.LinearLoss(tahq.make_loss_config(40, 64, 300, KINDS[kind][0], reduction=tahq.LOSS_SUM))
    loss.forward(big, weight, target)
    want, _ = loss64.forward(big, weight, target, IGNORE)
    assert ((loss.losses.double() - want).abs() <= 1e-4 * (1 + big.double().abs() @ weight.double().abs().t().amax(1))).all()
    y = x.abs()
    masked = weight.clone()
    masked[7] = float("-inf")
    target[target == 7] = 8
    loss.forward(y, masked, target)
    rest = torch.arange(300, device="cuda") != 7
    want, _ = loss64.forward(y, masked[rest], torch.where(target > 7, target - 1, target), IGNORE)
    off, lse_off, _ = _bounds(y, masked[rest], target, kind)
    assert ((loss.losses.double() - want).abs() <= off + lse_off + UNIT * want.abs()).all()
    y[5, 3] = float("nan")
    loss.forward(y, weight, target)
    nan = torch.arange(40, device="cuda") == 5
    assert loss.losses[nan].isnan().all() and loss.losses[~nan].isfinite().all()


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("counted", (0, 1, 5))
def test_infinite_weights_and_rows_that_are_no_tokens(kind, counted):
    """Products with a row of -infinity are -infinity or, of zeros, NaN: where fewer tokens count than a stage has rows, what fills it up adds nothing
    to the weight's gradient, that row's neither."""
    x, weight, target, _ = _make(40, 64, 300, kind, 0.0)
    weight[7] = float("-inf")
    x, target = x.abs() + 0.5, torch.where(target == 7, 8, target)
    target[counted:] = IGNORE
    loss = tahq.LinearLoss(tahq.make_loss_config(40, 64, 300, KINDS[kind][0], reduction=tahq.LOSS_SUM))
    loss.forward(x, weight, target)
    _, grad_w = loss.backward(x, weight, target)
    assert grad_w.isfinite().all() and (grad_w[7] == 0).all() and (counted == 0) == bool((grad_w == 0).all())


def test_class_slots_streams_and_refusals():
    rows, cols, vocab = 70, 64, 300
    loss = tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, tahq.BF16), in_flight=2)
    sets = [_make(rows, cols, vocab, "bf16", seed=s)[:3] for s in (1, 2)]
    alone = []
    for s in sets:
        one = tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, tahq.BF16))
        alone.append((one.forward(*s).clone(), *(t.clone() for t in one.backward(*s))))
    with pytest.raises(ValueError):
        loss.backward(*sets[0])
    totals = [loss.forward(*s, slot=i) for i, s in enumerate(sets)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in (1, 0):
        grads = loss.backward(*sets[i], stream=side, slot=i)
        side.synchronize()
        assert torch.equal(totals[i], alone[i][0]) and torch.equal(grads[0], alone[i][1]) and torch.equal(grads[1], alone[i][2])
    half = torch.full((1,), 0.5, device="cuda")
    assert torch.equal(loss.backward(*sets[0], grad_loss=half)[1], (alone[0][2].float() / 2).bfloat16())
    x, weight, target = sets[0]
    for bad in ((x.float(), weight, target), (x[:69], weight, target), (x, weight[:, :63], target), (x, weight, target.int()), (x, weight, target[:5]),
                (x.view(64, 70), weight, target), (x.cpu(), weight, target), (x, weight.t().contiguous().t(), target)):
        with pytest.raises(ValueError):
            loss.forward(*bad)
    with pytest.raises(ValueError):
        tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, tahq.BF16), training=False).backward(*sets[0])
    frozen = tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, tahq.BF16), frozen=True)
    frozen.forward(*sets[0])
    grads = frozen.backward(*sets[0])
    assert grads[1] is None and torch.equal(grads[0], alone[0][1])
    each = tahq.LinearLoss(tahq.make_loss_config(rows, cols, vocab, tahq.BF16, reduction=tahq.LOSS_NONE))
    assert each.forward(*sets[0]).shape == (rows,)


def test_graph_replays():
    """A captured forward and backward pass, replayed on other numbers and other counts of tokens, with eager work in between."""
    rows, cols, vocab = 300, 96, 1100
    x, weight, target, _ = _make(rows, cols, vocab, "bf16")
    cfg = tahq.make_loss_config(rows, cols, vocab, tahq.BF16)
    captured, eager = tahq.LinearLoss(cfg), tahq.LinearLoss(cfg)
    captured.forward(x, weight, target), captured.backward(x, weight, target)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        total = captured.forward(x, weight, target)
        grads = captured.backward(x, weight, target)
    for replay in range(4):
        other = _make(rows, cols, vocab, "bf16", 0.2 * replay, seed=10 + replay)
        for t, v in zip((x, weight, target), other):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(total, eager.forward(x, weight, target)) and all(torch.equal(a, b) for a, b in zip(grads, eager.backward(x, weight, target)))
