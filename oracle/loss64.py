"""Softmax cross entropy over a vocabulary in 64 bits (include/tahq_loss.h), forward and backward.  Tensors may be on any device."""
import torch


def forward(x, weight, target, ignore):
    """(losses, lse) of every token, zeros for those that do not count, NaN for a target that is none."""
    vocab = weight.shape[0]
    counts = target != ignore
    logits = x.double() @ weight.double().t()
    lse = torch.logsumexp(logits, 1)
    good = (target >= 0) & (target < vocab)
    at = logits.gather(1, target.clamp(0, vocab - 1)[:, None])[:, 0]
    losses = torch.where(good, lse - at, torch.full_like(lse, float("nan")))
    zero = torch.zeros_like(lse)
    return torch.where(counts, losses, zero), torch.where(counts, lse, zero)


def reduced(losses, target, ignore, reduction):
    n = int((target != ignore).sum())
    return losses.sum() / (max(n, 1) if reduction == 2 else 1), n


def grads_of_logits(x, weight, target, ignore):
    """p - [v = t], zeros for tokens that do not count."""
    logits = x.double() @ weight.double().t()
    p = torch.softmax(logits, 1)
    counts = target != ignore
    rows = torch.arange(x.shape[0], device=x.device)[counts]
    p[rows, target[counts]] -= 1
    return torch.where(counts[:, None], p, torch.zeros_like(p))


def backward(x, weight, target, ignore, g):
    """g: gradient of every token's loss (those that do not count: any)."""
    d = grads_of_logits(x, weight, target, ignore) * torch.where(target != ignore, g, torch.zeros_like(g))[:, None]
    x0 = torch.where((target != ignore)[:, None], x.double(), torch.zeros_like(x, dtype=torch.float64))
    return d @ weight.double(), d.t().contiguous() @ x0, d
