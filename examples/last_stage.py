"""One training step of a pipeline's last stage: activations come in, a block with attention, the loss over the vocabulary, and everything back.

    python examples/last_stage.py [--batch 2] [--seq 128] [--hidden 512] [--heads 8] [--k-heads 2] [--vocab 5003] [--dtype bf16]

Forward    the boundary's activations are decoded; h = RMSNorm(r) w_pre; one packed projection to queries, keys and values; queries and keys normed head by
           head and rotated by position in one pass; causal attention and its projection (torch, fp32); r' = r + dropout(block); hf = RMSNorm(r') w_final;
           loss = mean over the tokens that count of cross entropy(hf W^T), a quarter of every sample being a prompt that does not
Backward   gradients of hf and W without the logits; through the norm, the dropout's mask, attention, the rotation and the heads' norms into the packed
           projection's gradient; through the first norm to the received activations, encoded by the 8-bit fixed-point codec

Prints the loss and every result's distance from the same step in 64 bits (2-norm of the difference over that of the result)."""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2506_01352_amd as tahq  # noqa: E402

EPS, BASE, P, GRADIENT_SCALE = 1e-6, 10000.0, 0.1, 2.0 ** 14


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def attention(q, k, v, batch, seq):
    """Causal attention in the inputs' precision: [tokens, heads, head], every key head for a run of query heads."""
    shape = lambda t: t.unflatten(0, (batch, seq)).transpose(1, 2)      # noqa: E731
    each = q.shape[1] // k.shape[1]
    q, k, v = shape(q), *(shape(t).repeat_interleave(each, 1) for t in (k, v))
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * q.shape[-1] ** -0.5
    hidden = torch.ones(seq, seq, dtype=torch.bool, device=q.device).triu(1)
    weights = torch.softmax(scores.masked_fill(hidden, float("-inf")), -1)
    return torch.matmul(weights, v.contiguous()).transpose(1, 2).flatten(2).flatten(0, 1)


def step64(t, target, positions, mask, batch, seq, q_heads, k_heads, ignore):
    """The same step in 64 bits by autograd: loss and gradients."""
    t = {n: v.double().detach().requires_grad_() for n, v in t.items()}
    norm = lambda v, w: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * w      # noqa: E731
    h = norm(t["r"], t["w_pre"])
    qkv = h @ t["w_qkv"].t()
    head = t["w_q"].shape[0]
    q, k, v = (p.unflatten(1, (-1, head)) for p in qkv.split([q_heads * head, k_heads * head, k_heads * head], 1))
    angle = positions.double()[:, None, None] * BASE ** (-torch.arange(0, head, 2, device=q.device).double() / head)

    def turned(x):
        a, b = x[..., :head // 2], x[..., head // 2:]
        return torch.cat((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1)

    block = attention(turned(norm(q, t["w_q"])), turned(norm(k, t["w_k"])), v, batch, seq) @ t["w_o"].t()
    hf = norm(t["r"] + block * mask.double(), t["w_final"])
    counts = target != ignore
    loss = torch.nn.functional.cross_entropy((hf @ t["w_vocab"].t())[counts], target[counts])
    loss.backward()
    return float(loss.detach()), {n: v.grad for n, v in t.items()}


def run(batch=2, seq=128, hidden=512, heads=8, k_heads=2, vocab=5003, seed=3, dtype="bf16", mask=None):
    """mask: [tokens * hidden], which elements the dropout under `seed`, offset 0, is to keep, for the step in 64 bits; None: what its backward pass keeps."""
    tokens, head, ignore = batch * seq, hidden // heads, -100
    kind, storage = {"bf16": (tahq.BF16, torch.bfloat16), "f32": (tahq.F32, torch.float32)}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(storage)      # noqa: E731
    wide = (heads + 2 * k_heads) * head
    w = {"w_pre": 1 + 0.1 * normal(hidden), "w_qkv": normal(wide, hidden) * hidden ** -0.5, "w_q": 1 + 0.1 * normal(head), "w_k": 1 + 0.1 * normal(head),
         "w_o": normal(hidden, heads * head) * hidden ** -0.5, "w_final": 1 + 0.1 * normal(hidden), "w_vocab": normal(vocab, hidden) * hidden ** -0.5}
    positions = torch.arange(tokens, device="cuda") % seq
    target = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    target[positions < seq // 4] = ignore

    # ---- forward
    codec = tahq.Codec(tahq.make_config(batch, seq, hidden, 64, kind, 3.8))
    codec.encode(normal(tokens, hidden))
    r = codec.decode().view(tokens, hidden)
    norm_cfg = tahq.make_norm_config(tokens, hidden, kind, eps=EPS)
    pre, final = tahq.BlockNorm(norm_cfg), tahq.BlockNorm(norm_cfg)
    _, h = pre.forward(r, None, None, None, w["w_pre"])
    qkv = h @ w["w_qkv"].t()
    views = lambda t: tuple(p.unflatten(1, (-1, head)) for p in t.split([heads * head, k_heads * head, k_heads * head], 1))      # noqa: E731
    q, k, v = views(qkv)
    rotary = tahq.HeadRotary(tahq.make_heads_config(tokens, heads, k_heads, head, head, kind, eps=EPS, ldq=wide, ldk=wide), tahq.make_rotary_config(head, BASE))
    q_turned, k_turned = rotary.forward(q, k, w["w_q"], w["w_k"], positions)
    leaves = [t.detach().requires_grad_() for t in (q_turned, k_turned, v, w["w_o"])]
    block = attention(*(t.float() for t in leaves[:3]), batch, seq).to(storage) @ leaves[3].t()
    drop = tahq.Dropout(tahq.make_dropout_config(tokens * hidden, kind, P, seed=seed))
    r_out = drop.forward(block.detach(), r)
    _, hf = final.forward(r_out, None, None, None, w["w_final"])
    head_loss = tahq.LinearLoss(tahq.make_loss_config(tokens, hidden, vocab, kind, ignore=ignore))
    loss = head_loss.forward(hf, w["w_vocab"], target)

    # ---- backward
    grads = {}
    grad_hf, grads["w_vocab"] = head_loss.backward(hf, w["w_vocab"], target)
    back = final.backward(None, grad_hf, None, None, None, r_out, w["w_final"], final.stats)
    grads["w_final"], grad_r = back["grad_w_pre"], back["grad_residual"]
    grad_block = drop.backward(grad_r)
    grad_q, grad_k, grad_v, grads["w_o"] = torch.autograd.grad(block, leaves, grad_block)
    grad_qkv = torch.empty_like(qkv)
    views(grad_qkv)[2].copy_(grad_v)
    got = rotary.backward(grad_q.contiguous(), grad_k.contiguous(), q, k, w["w_q"], w["w_k"], positions, out=views(grad_qkv)[:2])
    grads["w_q"], grads["w_k"] = got["grad_w_q"], got["grad_w_k"]
    grads["w_qkv"] = grad_qkv.t() @ h
    back = pre.backward(grad_r, grad_qkv @ w["w_qkv"], None, None, None, r, w["w_pre"], pre.stats)
    grads["w_pre"], grads["r"] = back["grad_w_pre"], back["grad_residual"]
    naive = tahq.make_naive_config(batch, seq, hidden, kind, 8, GRADIENT_SCALE)
    wire = torch.empty(tahq.tahq_naive_packed_size(naive), dtype=torch.uint8, device="cuda")
    tahq.tahq_naive_encode(naive, grads["r"], wire)

    # ---- the same in 64 bits, with the same mask
    kept = drop.backward(torch.ones_like(r)) != 0 if mask is None else mask.to(r.device).view(r.shape)
    mask = torch.where(kept, 65536 / (65536 - round(65536 * P)), 0.0)
    torch.cuda.synchronize()
    want_loss, want = step64({"r": r, **w}, target, positions, mask, batch, seq, heads, k_heads, ignore)
    return {"loss": float(loss), "loss64": want_loss, "wire": wire.numel(), "errors": {n: off(grads[n], want[n]) for n in want}}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 2), ("seq", 128), ("hidden", 512), ("heads", 8), ("k-heads", 2), ("vocab", 5003)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    got = run(**vars(ap.parse_args()))
    print(f"loss {got['loss']:.5f}, in 64 bits {got['loss64']:.5f}; gradient on the wire {got['wire']} bytes")
    for name, value in got["errors"].items():
        print(f"gradient of {name:8s} off by {value:.1e}")


if __name__ == "__main__":
    main()
