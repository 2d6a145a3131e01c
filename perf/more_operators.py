"""Performance cases of what else a stage of a transformer runs in training: per-head norms and rotary positions of queries and keys,
dropout in front of the residual, and at the last stage the loss over the vocabulary, from the hidden states to the gradients.

A case is a plain dict:
  kind     "heads"      queries and keys behind their projection: normed head by head (norm 1), rotated by position   (forward)
           "headsgrad"  gradients of queries, keys and the norms' weights                                              (backward)
           "dropout"    residual + dropped(x): the mask comes from a counter and is never stored                       (forward)
           "dropgrad"   the same mask on the gradient                                                                  (backward)
           "loss"       cross entropy of hidden states against a vocabulary's weight, no gradients                     (evaluation)
           "lossgrad"   the same and the gradients of hidden states and weight, logits not kept                        (training)
  dtype    "bf16" or "f32": storage type of activations, weights and gradients; sums, statistics and the norms' weights' gradients are fp32
  heads    q_heads, k_heads, head: channels of a head, rotated: how many of them are, pairs: 1 = channels (2i, 2i + 1) are a pair, 0 =
           (i, i + rotated / 2); packed: 1 = queries and keys are views of one [tokens, (q + 2 k) head] tensor
  scaling  "plain", "linear" (positions / factor), "stretched" (larger base), "parts" (slow channels / factor, fast ones as they are)
  start    position of the first token; tokens of a sample follow each other, every sample begins at `start`
  p        probability to drop
  rows, cols, vocab    tokens, channels, rows of the vocabulary's weight
  ignored  tokens at the head of each of `samples` samples whose target is "ignore" (a prompt, say)

Where `own` is false, run() computes the same in elementary operations of 32 bits (angles in 64)."""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_EPS = 1e-6
_BASE, _ORIGINAL, _LOW, _HIGH = 10000.0, 4096, 1.0, 32.0
_IGNORE = -100


def _heads(kind, dtype, tokens, q_heads, k_heads, head, rotated, **more):
    c = {"kind": kind, "dtype": dtype, "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "head": head, "rotated": rotated,
         "pairs": 0, "norm": 1, "packed": 1, "scaling": "plain", "factor": 1.0, "start": 0, "samples": 1}
    return {**c, **more}


def _dropout(kind, dtype, rows, cols, p):
    return {"kind": kind, "dtype": dtype, "rows": rows, "cols": cols, "p": p}


def _loss(kind, dtype, rows, cols, vocab, ignored=0, samples=1):
    return {"kind": kind, "dtype": dtype, "rows": rows, "cols": cols, "vocab": vocab, "ignored": ignored, "samples": samples}


def _named(name, c):
    return {"name": name, **c}


def listed():
    return [
        # One decoding token far into a long context, grouped key heads: latency is all of it.
        _named("heads_bf16_1x32+8x128", _heads("heads", "bf16", 1, 32, 8, 128, 128, scaling="parts", factor=8.0, start=30001)),
        # A small fp32 model (25 heads of 64) without norms, half of each head rotated in pairs, far positions of a long text.
        _named("heads_f32_777x25+25x64_pairs", _heads("heads", "f32", 777, 25, 25, 64, 32, pairs=1, norm=0, scaling="linear", factor=4.0,
                                                       start=900001)),
        # All tokens of the repository's 5120-channel micro-batch (16 x 2048), 40 heads of 128 and 8 of keys, out of one packed projection.
        _named("heads_bf16_32768x40+8x128", _heads("heads", "bf16", 32768, 40, 8, 128, 128, samples=16)),
        # Its backward pass.
        _named("headsgrad_bf16_32768x40+8x128", _heads("headsgrad", "bf16", 32768, 40, 8, 128, 128, samples=16)),
        # An odd fp32 micro-batch (3 x 777 tokens) of heads of 80 channels of which 40 are rotated.
        _named("headsgrad_f32_2331x20+5x80", _heads("headsgrad", "f32", 2331, 20, 5, 80, 40, packed=0, scaling="stretched", factor=2.0, samples=3)),
        # The residual stream of the headline configuration's micro-batch (8 x 4096 tokens x 8192 channels).
        _named("dropout_bf16_32768x8192", _dropout("dropout", "bf16", 32768, 8192, 0.1)),
        # One sequence of a small model: a launch's time counts.
        _named("dropout_bf16_128x512", _dropout("dropout", "bf16", 128, 512, 0.1)),
        # Backward of an odd fp32 micro-batch.
        _named("dropgrad_f32_2331x1600", _dropout("dropgrad", "f32", 2331, 1600, 0.25)),
        # Five tokens scored against a vocabulary of 50257 by a model of 1600 channels: the weight's bytes are all of it.
        _named("loss_bf16_5x1600x50257", _loss("loss", "bf16", 5, 1600, 50257)),
        # Odd sizes throughout in fp32, the first 40 tokens of each of three samples ignored.
        _named("lossgrad_f32_333x1001x32003", _loss("lossgrad", "f32", 333, 1001, 32003, 40, 3)),
        # A micro-batch of two samples of the 1600-channel model, prompts of 300 tokens ignored.
        _named("lossgrad_bf16_2048x1600x50257", _loss("lossgrad", "bf16", 2048, 1600, 50257, 300, 2)),
        # The repository's 4096-channel configuration (8 x 1024 tokens) with a large vocabulary.
        _named("lossgrad_bf16_8192x4096x131072", _loss("lossgrad", "bf16", 8192, 4096, 131072)),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any kind; 1 to 32768 tokens; heads of 16 to 256 channels; 257 to 8191 channels and vocabularies of 1000 to 131072, odd
    ones among them; both types, all options."""
    kind = rng.choice(["heads", "headsgrad", "dropout", "dropgrad", "loss", "lossgrad", "lossgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = _BYTES[dtype]
    if kind in ("heads", "headsgrad"):
        head = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256, 2 * rng.randint(8, 128)])
        rotated = rng.choice([head, head, head, head // 4 * 2, head // 8 * 2])
        k_heads = rng.choice([1, 2, 4, 8])
        q_heads = k_heads * rng.choice([1, 2, 4, 5])
        top = (400 << 20) // ((q_heads + 2 * k_heads) * head * es)
        scaling = rng.choice(["plain", "linear", "stretched", "parts"])
        return _heads(kind, dtype, _log_uniform(rng, 1, min(32768, top)), q_heads, k_heads, head, rotated, pairs=rng.randint(0, 1),
                      norm=rng.randint(0, 3) > 0 and 1 or 0, packed=rng.randint(0, 1), scaling=scaling,
                      factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0, 3.7]), start=rng.choice([0, rng.randint(0, 1 << 20)]),
                      samples=rng.choice([1, 2, 3]))
    cols = rng.choice([512, 768, 1024, 1600, 2048, 2560, 4096, 5120, 8192]) if rng.random() < 0.7 else rng.randint(257, 8191)
    if kind in ("dropout", "dropgrad"):
        return _dropout(kind, dtype, _log_uniform(rng, 1, min(32768, (1 << 28) // cols // (es // 2))), cols, rng.choice([0.05, 0.1, 0.25, 0.5]))
    vocab = rng.choice([32000, 50257, 65536, 131072]) if rng.random() < 0.6 else _log_uniform(rng, 1000, 131071)
    top = (1 << 42) // (cols * vocab) // (1 if kind == "lossgrad" and dtype == "bf16" else 8)
    rows = _log_uniform(rng, 1 if kind == "loss" else 64, max(65, min(8192, top)))
    samples = rng.choice([1, 2, 3])
    return _loss(kind, dtype, rows, cols, vocab, rng.choice([0, 0, rows // samples // 3]), samples)


# ---------------------------------------------------------------- the operators in elementary operations

def _radians_per_position(c):
    """Angle that one position turns each pair by, in 64 bits."""
    half, base, s = c["rotated"] // 2, _BASE, c["factor"]
    if c["scaling"] == "stretched" and c["rotated"] > 2:
        base = base * s ** (c["rotated"] / (c["rotated"] - 2))
    f = base ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(half, 1))
    if c["scaling"] == "linear":
        f = f / s
    if c["scaling"] == "parts":
        kept = ((f * _ORIGINAL / (2 * math.pi) - _LOW) / (_HIGH - _LOW)).clamp(0, 1)
        f = kept * f + (1 - kept) * f / s
    return f


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


def _turned(x, cos, sin, c):
    """[tokens, heads, head]: the first `rotated` channels in pairs, the others as they are; -sin turns back."""
    r = c["rotated"]
    if c["pairs"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _cos_sin(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * _radians_per_position(c)[None]
    return (torch.cos(angle) * _magnitude(c)).float()[:, None], (torch.sin(angle) * _magnitude(c)).float()[:, None]


def _heads_forward(s):
    c = s["case"]
    cos, sin = _cos_sin(s)
    out = {}
    for n in ("q", "k"):
        x = s[n].float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * s["w_" + n].float()
        out[n] = _turned(x, cos, sin, c).to(s[n].dtype)
    return out


def _heads_backward(s):
    c = s["case"]
    cos, sin = _cos_sin(s)
    out = {}
    for n in ("q", "k"):
        g = _turned(s["grad_" + n].float(), cos, -sin, c)
        if c["norm"]:
            x = s[n].float()
            rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
            unit = x * rstd
            out["grad_w_" + n] = (g * unit).sum((0, 1))
            u = g * s["w_" + n].float()
            g = rstd * (u - unit * (u * unit).mean(-1, keepdim=True))
        out["grad_" + n] = g.to(s[n].dtype)
    return out


def _words(seed, offset, blocks):
    """The counter-based generator (Philox 4x32, ten rounds) at counters (block, offset) under key `seed`: four words of each block."""
    m = 0xFFFFFFFF
    block = torch.arange(blocks, dtype=torch.int64, device="cuda")
    c = [block & m, block >> 32, torch.full_like(block, offset & m), torch.full_like(block, offset >> 32)]
    key = [seed & m, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & m) ^ c[1] ^ key[0], b & m, (a >> 32 & m) ^ c[3] ^ key[1], a & m]
        key = [key[0] + 0x9E3779B9 & m, key[1] + 0xBB67AE85 & m]
    return torch.stack(c, 1)


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _dropped(x, s):
    """x where it is kept, times 1 / (1 - p): 16 bits an element, eight elements a block, p in steps of 2^-16."""
    t = _threshold(s["case"]["p"])
    words = _words(s["key"], s["offset"], -(-x.numel() // 8))
    bits = torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)[:x.numel()].view(x.shape)
    return torch.where(bits >= t, x.float() * (65536 / (65536 - t)), 0.0)


def _loss_forward(s):
    """losses and log-sum-exp of every token, their mean over those that count; and what the gradients start from."""
    logits = torch.matmul(s["x"].float(), s["weight"].float().t())
    counts = s["target"] != _IGNORE
    top = logits.amax(1)
    lse = top + (logits - top[:, None]).exp_().sum(1).log()
    at_target = logits.gather(1, s["target"].clamp_min(0)[:, None])[:, 0]
    losses = torch.where(counts, lse - at_target, 0.0)
    lse = torch.where(counts, lse, 0.0)
    return logits, counts, losses, lse, losses.sum() / counts.sum().clamp_min(1)


def _loss_backward(s, logits, counts, lse):
    each = counts.float() / counts.sum().clamp_min(1)
    g = logits.sub_(lse[:, None]).exp_()
    g[torch.arange(g.shape[0], device=g.device), s["target"].clamp_min(0)] -= 1.0
    g.mul_(each[:, None])
    return torch.matmul(g, s["weight"].float()).to(s["x"].dtype), torch.matmul(g.t(), s["x"].float()).to(s["weight"].dtype)


# ---------------------------------------------------------------- what a program has in hand

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(g, rows, cols, dtype):
    """N(0, 1) with a few channels x20, tokens of unlike size."""
    x = _normal(g, rows, cols)
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    x *= torch.exp(0.5 * _normal(g, rows, 1))
    return x.to(_TORCH[dtype])


def _gradients(g, rows, cols, dtype):
    """Activation gradients: around 1e-5, tokens of unlike size."""
    return (_normal(g, rows, cols) * 1e-5 * torch.exp(_normal(g, rows, 1))).to(_TORCH[dtype])


def _inputs(case, seed):
    """The tensors of a case, the same ones for run() and exact()."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    kind, dtype = case["kind"], case["dtype"]
    s = {"case": case}
    if kind in ("heads", "headsgrad"):
        t, hq, hk, d = case["tokens"], case["q_heads"], case["k_heads"], case["head"]
        if case["packed"]:
            x = _activations(g, t, (hq + 2 * hk) * d, dtype)
            s["q"], s["k"] = x[:, :hq * d].view(t, hq, d), x[:, hq * d:(hq + hk) * d].view(t, hk, d)
        else:
            s["q"], s["k"] = _activations(g, t, hq * d, dtype).view(t, hq, d), _activations(g, t, hk * d, dtype).view(t, hk, d)
        s["w_q"] = s["w_k"] = None
        if case["norm"]:
            s["w_q"], s["w_k"] = ((1 + 0.1 * _normal(g, d)).to(_TORCH[dtype]) for _ in range(2))
        each = -(-t // case["samples"])
        s["positions"] = case["start"] + torch.arange(t, device="cuda") % each
        if kind == "headsgrad":
            s["grad_q"], s["grad_k"] = _gradients(g, t, hq * d, dtype).view(t, hq, d), _gradients(g, t, hk * d, dtype).view(t, hk, d)
        return s
    rows, cols = case["rows"], case["cols"]
    if kind in ("dropout", "dropgrad"):
        s["x"] = (_activations if kind == "dropout" else _gradients)(g, rows, cols, dtype)
        if kind == "dropout":
            s["residual"] = _activations(g, rows, cols, dtype)
        s["key"], s["offset"] = int(seed) * 0x9E3779B97F4A7C1 % (1 << 63), int(seed) % 1000 + 1
        return s
    # hidden states behind the last norm, which lean towards their target's row for most tokens, as a trained model's do
    vocab = case["vocab"]
    weight = _normal(g, vocab, cols) * cols ** -0.5
    target = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    lean = 12.0 * torch.rand(rows, 1, generator=g, device="cuda") * (torch.rand(rows, 1, generator=g, device="cuda") < 0.7)
    s["x"] = (_normal(g, rows, cols) + lean * weight[target]).to(_TORCH[dtype])
    s["weight"] = weight.to(_TORCH[dtype])
    each = -(-rows // case["samples"])
    s["target"] = torch.where(torch.arange(rows, device="cuda") % each < case["ignored"], _IGNORE, target)
    return s


def prepare(case, seed):
    """Inputs, and the handle that a program keeps in between calls: buffers and the table of the rotation's frequencies."""
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2506_01352_amd as tahq
    kind, storage = case["kind"], {"f32": tahq.F32, "bf16": tahq.BF16}[case["dtype"]]
    if kind in ("heads", "headsgrad"):
        scaling = {"plain": tahq.ROTARY_PLAIN, "linear": tahq.ROTARY_LINEAR, "stretched": tahq.ROTARY_STRETCHED, "parts": tahq.ROTARY_PARTS}
        rotary = tahq.make_rotary_config(case["rotated"], _BASE, scaling[case["scaling"]], case["factor"], _ORIGINAL, _LOW, _HIGH)
        ld = (case["q_heads"] + 2 * case["k_heads"]) * case["head"] if case["packed"] else 0
        cfg = tahq.make_heads_config(case["tokens"], case["q_heads"], case["k_heads"], case["head"], case["rotated"], storage,
                                     layout=tahq.HEADS_PAIRS if case["pairs"] else tahq.HEADS_HALVES, norm=case["norm"], eps=_EPS,
                                     magnitude=_magnitude(case), ldq=ld, ldk=ld)
        s["heads"] = tahq.HeadRotary(cfg, rotary, training=kind == "headsgrad")
        if kind == "headsgrad":
            # gradients go to their places in the packed projection's, as the queries and keys came from there
            t, hq, hk, d = case["tokens"], case["q_heads"], case["k_heads"], case["head"]
            if case["packed"]:
                x = torch.zeros(t, ld, dtype=_TORCH[case["dtype"]], device="cuda")
                s["to"] = x[:, :hq * d].view(t, hq, d), x[:, hq * d:(hq + hk) * d].view(t, hk, d)
            else:
                s["to"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    elif kind in ("dropout", "dropgrad"):
        s["drop"] = tahq.Dropout(tahq.make_dropout_config(case["rows"] * case["cols"], storage, case["p"], s["key"]))
    else:
        cfg = tahq.make_loss_config(case["rows"], case["cols"], case["vocab"], storage, reduction=tahq.LOSS_MEAN, ignore=_IGNORE)
        s["loss"] = tahq.LinearLoss(cfg, training=kind == "lossgrad")
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        if kind == "heads":
            q, k = s["heads"].forward(s["q"], s["k"], s["w_q"], s["w_k"], s["positions"])
            return {"q": q, "k": k}
        if kind == "headsgrad":
            got = s["heads"].backward(s["grad_q"], s["grad_k"], s["q"], s["k"], s["w_q"], s["w_k"], s["positions"], out=s["to"])
            return {k: v for k, v in got.items() if v is not None}
        if kind == "dropout":
            return s["drop"].forward(s["x"], s["residual"], offset=s["offset"])
        if kind == "dropgrad":
            return s["drop"].backward(s["x"], offset=s["offset"])
        loss = s["loss"].forward(s["x"], s["weight"], s["target"])
        out = {"loss": loss, "losses": s["loss"].losses, "lse": s["loss"].lse}
        if kind == "lossgrad":
            out["grad_x"], out["grad_weight"] = s["loss"].backward(s["x"], s["weight"], s["target"])
        return out
    if kind == "heads":
        return _heads_forward(s)
    if kind == "headsgrad":
        return _heads_backward(s)
    if kind == "dropout":
        return (s["residual"].float() + _dropped(s["x"], s)).to(s["x"].dtype)
    if kind == "dropgrad":
        return _dropped(s["x"], s).to(s["x"].dtype)
    logits, counts, losses, lse, loss = _loss_forward(s)
    out = {"loss": loss.view(1), "losses": losses, "lse": lse}
    if kind == "lossgrad":
        out["grad_x"], out["grad_weight"] = _loss_backward(s, logits, counts, lse)
    return out


def _counted(case):
    """Tokens that are not ignored."""
    each = -(-case["rows"] // case["samples"])
    whole, rest = divmod(case["rows"], each)
    return whole * (each - min(case["ignored"], each)) + max(rest - case["ignored"], 0)


def work(case):
    kind, es = case["kind"], _BYTES[case["dtype"]]
    if kind in ("heads", "headsgrad"):
        elements = case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["head"]
        if kind == "heads":
            return {"bytes": 2 * elements * es + 8 * case["tokens"], "flops": (4 + 4 * case["norm"]) * elements}
        return {"bytes": (2 + case["norm"]) * elements * es + 8 * case["tokens"], "flops": (4 + 14 * case["norm"]) * elements}
    if kind in ("dropout", "dropgrad"):
        return {"bytes": (3 if kind == "dropout" else 2) * case["rows"] * case["cols"] * es, "flops": 15 * case["rows"] * case["cols"]}
    rows, cols, vocab, n = case["rows"], case["cols"], case["vocab"], _counted(case)
    if kind == "loss":
        return {"bytes": (n * cols + vocab * cols) * es + 16 * rows, "flops": 2 * n * cols * vocab}
    return {"bytes": (n * cols + rows * cols + 2 * vocab * cols) * es + 16 * rows, "flops": 6 * n * cols * vocab}


# ---------------------------------------------------------------- the definitions in 64 bits

def _rotations(case, positions):
    """The rotation of every token as a complex number for each pair, magnitude included."""
    r, s = case["rotated"], case["factor"]
    f = torch.tensor([_BASE ** (-2.0 * i / r) if r else 0.0 for i in range(r // 2)], dtype=torch.float64, device="cuda")
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "stretched" and r > 2:
        f = torch.tensor([(_BASE * s ** (r / (r - 2))) ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float64, device="cuda")
    if case["scaling"] == "parts":
        turns = _ORIGINAL * f / (2 * math.pi)                       # in the context that the model was trained with
        slow, fast = turns <= _LOW, turns >= _HIGH
        between = (turns - _LOW) / (_HIGH - _LOW)
        f = torch.where(fast, f, torch.where(slow, f / s, f / s + between * (f - f / s)))
    angle = positions.double()[:, None] * f
    return torch.polar(torch.full_like(angle, _magnitude(case)), angle)[:, None]


def _rotate64(x, z, case):
    r, y = case["rotated"], x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["pairs"] else (slice(0, r // 2), slice(r // 2, r))
    turned = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def _kept64(case, key, offset, n):
    """Which elements are kept: Philox by 16-bit limbs, so that no product passes 2^63."""
    def product(a, constant):
        """High and low word of a 32-bit number times a 32-bit constant."""
        c1, c0, a1, a0 = constant >> 16, constant & 0xFFFF, a >> 16, a & 0xFFFF
        low = a0 * c0
        middle = a1 * c0 + (low >> 16)
        other = a0 * c1 + (middle & 0xFFFF)
        return a1 * c1 + (middle >> 16) + (other >> 16), (other & 0xFFFF) << 16 | low & 0xFFFF

    i = torch.arange(-(-n // 8), dtype=torch.int64, device="cuda")
    x0, x1, x2, x3 = i % (1 << 32), i // (1 << 32), torch.full_like(i, offset % (1 << 32)), torch.full_like(i, offset // (1 << 32))
    for turn in range(10):
        k0, k1 = (key % (1 << 32) + turn * 0x9E3779B9) % (1 << 32), (key // (1 << 32) + turn * 0xBB67AE85) % (1 << 32)
        h0, l0 = product(x0, 0xD2511F53)
        h1, l1 = product(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
    halves = [w // d % 65536 for w in (x0, x1, x2, x3) for d in (1, 65536)]
    return torch.stack(halves, 1).reshape(-1)[:n] >= _threshold(case["p"])


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "heads":
        z, out = _rotations(case, s["positions"]), {}
        for n in ("q", "k"):
            x = s[n].double()
            if case["norm"]:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["head"] + _EPS) * s["w_" + n].double()
            out[n] = _rotate64(x, z, case)
        return out
    if kind == "headsgrad":
        z, out = _rotations(case, s["positions"]).conj(), {}
        for n in ("q", "k"):
            g = _rotate64(s["grad_" + n].double(), z, case)
            if case["norm"]:
                x = s[n].double()
                size = torch.sqrt((x * x).sum(-1, keepdim=True) / case["head"] + _EPS)
                out["grad_w_" + n] = (g * x / size).sum((0, 1))
                u = g * s["w_" + n].double()
                g = u / size - x * ((u * x).sum(-1, keepdim=True) / (case["head"] * size ** 3))
            out["grad_" + n] = g
        return out
    if kind in ("dropout", "dropgrad"):
        x, t = s["x"].double(), _threshold(case["p"])
        kept = _kept64(case, s["key"], s["offset"], x.numel()).view(x.shape)
        out = x * kept * 65536 / (65536 - t)
        return out + s["residual"].double() if kind == "dropout" else out
    counts = (s["target"] != _IGNORE).nonzero()[:, 0]
    x, w, target = s["x"].double()[counts], s["weight"].double(), s["target"][counts]
    logits = torch.mm(x, w.t())
    lse = torch.logsumexp(logits, 1)
    n, m = case["rows"], max(len(counts), 1)
    every_lse, losses = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    every_lse[counts], losses[counts] = lse, lse - logits[torch.arange(len(counts), device="cuda"), target]
    out = {"loss": losses.sum().view(1) / m, "losses": losses, "lse": every_lse}
    if kind == "lossgrad":
        p = torch.softmax(logits, 1).div_(m)
        del logits
        p[torch.arange(len(counts), device="cuda"), target] -= 1.0 / m
        grad_x = torch.zeros(n, case["cols"], dtype=torch.float64, device="cuda")
        grad_x[counts] = torch.mm(p, w)
        out.update(grad_x=grad_x, grad_weight=torch.mm(p.t().contiguous(), x))
    return out
