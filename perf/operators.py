"""Performance cases of a pipeline stage's entry in 4 bits: microscaled 4-bit (mx4) quantization and product, and the norms
before and after a block fused with its gate and residual scale.

A case is a plain dict:
  kind     "linear"   y = x W^T, x quantized in the call, W kept in mx4                       (forward, down to a single token)
           "grad"     dx = dy W and dW = dy^T x of the same layer, dy quantized both ways in the call    (backward)
           "trip"     a tensor to mx4, along its rows and (both) along its columns, and back to values
           "norm"     r' = a r + g RMSNorm(b) w_post, h = RMSNorm(r') w_pre                   (forward)
           "normgrad" gradients of r, b, the gate and both weights                            (backward)
           "entry"    "norm" whose h goes to mx4 in the same pass, and the product y = h W^T  (a stage's entry)
  dtype    "bf16" or "f32": storage type of activations and their gradients
  rows     tokens; cols: channels; n: output features ("linear", "grad", "entry")
  transform  1: blocks of 32 are rotated by a Hadamard matrix before they are quantized
  cover    1: block scales never saturate; 0: they are 2^(floor(log2(max)) - 2)
  both     ("trip") 1: along rows and columns from one read
  gate_rows  tokens that share a row of the gate; 0: no gate

Where `own` is false, run() computes the same in elementary 32-bit operations."""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_EPS = 1e-6
_RESIDUAL_SCALE = 0.8125
_MX4_BYTES = 0.5 + 1 / 32


def _case(kind, dtype, rows, cols, **more):
    return {"kind": kind, "dtype": dtype, "rows": rows, "cols": cols, **more}


def _linear(kind, dtype, rows, cols, n, transform=0, cover=0, **more):
    return _case(kind, dtype, rows, cols, n=n, transform=transform, cover=cover, **more)


def _named(name, c):
    return {"name": name, **c}


def listed():
    return [
        # One token through a square projection of a GPT-2-XL-like model (1600 channels): latency is nearly all of it.
        _named("linear_bf16_1x1600x1600", _linear("linear", "bf16", 1, 1600, 1600)),
        # Five tokens (a small batch of decoding sequences) through a wide layer: the weights' bytes are all of it.
        _named("linear_bf16_5x8192x8192", _linear("linear", "bf16", 5, 8192, 8192, 0, 1)),
        # A prompt of odd length through the same small model's first feed-forward matrix.
        _named("linear_f32_777x1600x6400", _linear("linear", "f32", 777, 1600, 6400, 1, 1)),
        # Two samples of the headline configuration (4096 tokens x 8192 channels) through a square projection.
        _named("linear_bf16_8192x8192x8192", _linear("linear", "bf16", 8192, 8192, 8192)),
        # Backward of the small model's projection for a micro-batch of two samples: few tiles, a long sum over tokens.
        _named("grad_bf16_2048x1600x1600", _linear("grad", "bf16", 2048, 1600, 1600, 1, 1)),
        # Backward at the width of the repository's 4096-channel configuration, all 8 x 1024 tokens.
        _named("grad_bf16_8192x4096x8192", _linear("grad", "bf16", 8192, 4096, 8192, 0, 1)),
        # What training keeps of an activation: along channels for the product, along tokens for the weight's gradient.
        _named("trip_bf16_32768x8192_both", _case("trip", "bf16", 32768, 8192, transform=0, cover=0, both=1)),
        # A small fp32 model's activations with a width that is no multiple of anything.
        _named("trip_f32_2048x2047", _case("trip", "f32", 2048, 2047, transform=1, cover=1, both=0)),
        # One decoding token at the residual stream: two norms and a gate in one launch.
        _named("norm_bf16_1x4096", _case("norm", "bf16", 1, 4096, gate_rows=1)),
        # The residual stream of the repository's largest micro-batch by tokens, a gate per sample.
        _named("normgrad_bf16_32768x5120", _case("normgrad", "bf16", 32768, 5120, gate_rows=2048)),
        # A small model's odd micro-batch (3 x 777 tokens) in fp32, one gate for all tokens.
        _named("normgrad_f32_2331x1600", _case("normgrad", "f32", 2331, 1600, gate_rows=2331)),
        # A stage's entry: norms, gate and residual of 8 x 1024 tokens, h leaves the pass in mx4 and goes into the product.
        _named("entry_bf16_8192x4096x4096", _linear("entry", "bf16", 8192, 4096, 4096, 0, 1, gate_rows=1024)),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    """A model's width, or any other: odd ones among them."""
    if rng.random() < 0.7:
        return rng.choice([512, 768, 1024, 1600, 2048, 2560, 4096, 5120, 8192])
    return rng.randint(257, 8191)


def draw(rng):
    """One more case: any kind, 1 to 32768 tokens, widths of 257 to 8192, both types, all options."""
    kind = rng.choice(["linear", "linear", "linear", "grad", "grad", "trip", "norm", "normgrad", "entry"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    cols, n = _width(rng), _width(rng)
    transform, cover = rng.randint(0, 1), rng.randint(0, 1)
    if kind in ("linear", "entry", "grad"):
        # few tokens as often as many; no more products than the largest listed case
        top = (1 << 39) // (cols * n) // (2 if kind == "grad" else 1)
        rows = _log_uniform(rng, 16 if kind == "grad" else 1, min(16384, top))
        c = _linear(kind, dtype, rows, cols, n, transform, cover)
    else:
        top = (1 << 28) // cols // (2 if dtype == "f32" else 1)
        rows = _log_uniform(rng, 1, min(32768, top))
        c = _case(kind, dtype, rows, cols)
        if kind == "trip":
            c.update(transform=transform, cover=cover, both=rng.randint(0, 1))
    if kind in ("norm", "normgrad", "entry"):
        c["gate_rows"] = rng.choice([0, rows, rows, max(1, -(-rows // rng.choice([2, 3, 8])))])
    return c


# ---------------------------------------------------------------- the operators in elementary 32-bit operations

_ROOT = 0.17677669529663687      # 1 / sqrt(32)


def _blocks(x):
    """[rows, cols] -> [rows, blocks, 32], the last block of a row filled with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % 32)).view(x.shape[0], -1, 32)


def _butterfly(y):
    """Sylvester's Hadamard matrix on the last axis of 32, times 1 / sqrt(32)."""
    shape = y.shape
    for h in (1, 2, 4, 8, 16):
        y = y.reshape(*shape[:-1], 16 // h, 2, h)
        a, b = y[..., 0, :], y[..., 1, :]
        y = torch.stack((a + b, a - b), -2)
    return y.reshape(shape) * torch.tensor(_ROOT, dtype=torch.float32, device=y.device)


def _mx4_values(x, transform, cover):
    """The values that a [rows, cols] tensor's mx4 form stands for, rotated blocks left rotated: [rows, 32 * blocks]."""
    y = _blocks(x.float())
    if transform:
        y = _butterfly(y)
    top = y.abs().amax(-1, keepdim=True).view(torch.int32)
    s = ((top + 0x3FFFFF if cover else top) >> 23).sub(2).clamp_min(0)
    scale = torch.where(s > 0, s << 23, 0x400000).to(torch.int32).view(torch.float32)
    a = y.abs() * ((254 - s) << 23).view(torch.float32)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.int32)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device)
    return (torch.copysign(grid[code], y) * scale).view(x.shape[0], -1)


def _mx4_trip(x, transform, cover):
    v = _mx4_values(x, transform, cover)
    if transform:
        v = _butterfly(v.view(v.shape[0], -1, 32)).view(v.shape)
    return v[:, :x.shape[1]].to(x.dtype)


def _gate_of_rows(gate, gate_rows, rows):
    return gate.float().repeat_interleave(gate_rows, 0)[:rows] if gate is not None else None


def _norm(s):
    c = s["case"]
    b, r = s["block"].float(), s["residual"].float()
    rstd_b = torch.rsqrt(b.square().mean(1) + _EPS)
    p = b * rstd_b[:, None] * s["w_post"].float()
    if s["gate"] is not None:
        p = p * _gate_of_rows(s["gate"], c["gate_rows"], c["rows"])
    out = r * _RESIDUAL_SCALE + p
    rstd_r = torch.rsqrt(out.square().mean(1) + _EPS)
    return out, out * rstd_r[:, None] * s["w_pre"].float(), torch.stack((rstd_b, rstd_r))


def _norm_grad(s):
    c, kind = s["case"], s["block"].dtype
    rstd_b, rstd_r = s["stats"][0][:, None], s["stats"][1][:, None]
    x1, x2 = s["block"].float() * rstd_b, s["residual_out"].float() * rstd_r
    dh, w_post = s["grad_h"].float(), s["w_post"].float()
    t = dh * s["w_pre"].float()
    g = s["grad_residual_out"].float() + rstd_r * (t - x2 * (t * x2).mean(1, keepdim=True))
    gated = g
    out = {}
    if s["gate"] is not None:
        groups = s["gate"].shape[0]
        each = torch.nn.functional.pad(g * x1 * w_post, (0, 0, 0, groups * c["gate_rows"] - c["rows"]))
        out["grad_gate"] = each.view(groups, c["gate_rows"], -1).sum(1)
        gated = g * _gate_of_rows(s["gate"], c["gate_rows"], c["rows"])
    u = gated * w_post
    out.update(grad_residual=(g * _RESIDUAL_SCALE).to(kind), grad_block=(rstd_b * (u - x1 * (u * x1).mean(1, keepdim=True))).to(kind),
               grad_w_post=(gated * x1).sum(0), grad_w_pre=(dh * x2).sum(0))
    return out


# ---------------------------------------------------------------- what a program has in hand

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(g, rows, cols, dtype):
    """N(0, 1) with a few channels x20, tokens of unlike size, one token in fifty all zero (padding)."""
    x = _normal(g, rows, cols)
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    x *= torch.exp(0.5 * _normal(g, rows, 1)) * (torch.rand(rows, 1, generator=g, device="cuda") > (0.02 if rows > 1 else 0.0))
    return x.to(_TORCH[dtype])


def _gradients(g, rows, cols, dtype):
    """Activation gradients: around 1e-5, tokens of unlike size, one element in a thousand x30."""
    x = _normal(g, rows, cols) * 1e-5 * torch.exp(_normal(g, rows, 1))
    x *= torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 0.001, 30.0, 1.0)
    return x.to(_TORCH[dtype])


def _inputs(case, seed):
    """The tensors of a case, the same ones for run() and exact()."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    kind, dtype, rows, cols = case["kind"], case["dtype"], case["rows"], case["cols"]
    s = {"case": case}
    if kind in ("linear", "grad", "entry"):
        s["weight"] = (_normal(g, case["n"], cols) * cols ** -0.5).to(_TORCH[dtype])
    if kind in ("linear", "trip", "grad"):
        s["x"] = _activations(g, rows, cols, dtype)
    if kind == "grad":
        s["grad_y"] = _gradients(g, rows, case["n"], dtype)
    if kind in ("norm", "entry", "normgrad"):
        s["residual"], s["block"] = _activations(g, rows, cols, dtype), _activations(g, rows, cols, dtype)
        s["w_post"], s["w_pre"] = ((1 + 0.1 * _normal(g, cols)).to(_TORCH[dtype]) for _ in range(2))
        s["gate"] = None
        if case["gate_rows"]:
            s["gate"] = (0.5 + 0.2 * _normal(g, -(-rows // case["gate_rows"]), cols)).to(_TORCH[dtype])
    if kind == "normgrad":
        s["grad_h"], s["grad_residual_out"] = _gradients(g, rows, cols, dtype), _gradients(g, rows, cols, dtype)
        out, _, s["stats"] = _norm(s)
        s["residual_out"] = out.to(_TORCH[dtype])
        del s["residual"]
    return s


def prepare(case, seed):
    """Inputs, and the handle with the layer's weights in the form that a program keeps them in between calls: mx4, or the same
    values in 32 bits for the plain form.  "grad" has the layer after its forward pass, which has kept x along tokens."""
    s = _inputs(case, seed)
    kind, rows, cols = case["kind"], case["rows"], case["cols"]
    options = (case.get("transform"), case.get("cover"))
    if not own:
        if kind in ("linear", "entry"):
            s["w_values"] = _mx4_values(s.pop("weight"), *options)
        if kind == "grad":
            s["w_values"] = _mx4_values(s.pop("weight").t().contiguous(), *options)
            s["x_values"] = _mx4_values(s.pop("x").t().contiguous(), *options)
        return s
    import paper_2506_01352_amd as tahq
    storage = {"f32": tahq.F32, "bf16": tahq.BF16}[case["dtype"]]
    kinds = {"transform": case.get("transform", 0), "scale_rule": case.get("cover", 0)}
    if kind in ("linear", "grad"):
        s["layer"] = tahq.Mx4Linear(s.pop("weight"), rows, training=kind == "grad", **kinds)
        if kind == "grad":
            s["layer"].forward(s.pop("x"))
    elif kind == "trip":
        s["trip"] = tahq.Mx4Tensor(tahq.make_mx4_config(rows, cols, storage, **kinds), transposed=bool(case["both"]))
    else:
        s["norm"] = tahq.BlockNorm(tahq.make_norm_config(rows, cols, storage, case["gate_rows"], _EPS, _RESIDUAL_SCALE, **kinds),
                                   mx4=kind == "entry")
        if kind == "entry":
            s["layer"] = tahq.Mx4Linear(s.pop("weight"), rows, **kinds)
    return s


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        if kind == "linear":
            return s["layer"].forward(s["x"])
        if kind == "grad":
            dx, dw = s["layer"].backward(s["grad_y"])
            return {"grad_x": dx, "grad_w": dw}
        if kind == "trip":
            s["trip"].quantize(s["x"])
            return s["trip"].dequantize()
        if kind == "norm":
            out, h = s["norm"].forward(s["residual"], s["block"], s["w_post"], s["gate"], s["w_pre"])
            return {"residual": out, "h": h, "stats": s["norm"].stats}
        if kind == "entry":
            out, h = s["norm"].forward(s["residual"], s["block"], s["w_post"], s["gate"], s["w_pre"])
            return {"residual": out, "y": s["layer"].product(h)}
        got = s["norm"].backward(s["grad_residual_out"], s["grad_h"], s["block"], s["w_post"], s["gate"], s["residual_out"],
                                 s["w_pre"], s["stats"])
        return {k: v for k, v in got.items() if v is not None}
    kept, options = _TORCH[c["dtype"]], (c.get("transform"), c.get("cover"))
    if kind == "linear":
        return torch.matmul(_mx4_values(s["x"], *options), s["w_values"].t()).to(kept)
    if kind == "grad":
        dy = s["grad_y"].float()
        dx = torch.matmul(_mx4_values(dy, *options), s["w_values"].t()).to(kept)
        return {"grad_x": dx, "grad_w": torch.matmul(_mx4_values(dy.t(), *options), s["x_values"].t())}
    if kind == "trip":
        rows = _mx4_trip(s["x"], *options)
        return (rows, _mx4_trip(s["x"].t(), *options)) if c["both"] else (rows,)
    if kind == "norm":
        out, h, stats = _norm(s)
        return {"residual": out.to(kept), "h": h.to(kept), "stats": stats}
    if kind == "entry":
        out, h, _ = _norm(s)
        return {"residual": out.to(kept), "y": torch.matmul(_mx4_values(h, *options), s["w_values"].t()).to(kept)}
    return _norm_grad(s)


def work(case):
    kind, rows, cols, es = case["kind"], case["rows"], case["cols"], _BYTES[case["dtype"]]
    n, elements = case.get("n", 0), rows * cols
    gate = cols * es * (-(-rows // case["gate_rows"]) if case.get("gate_rows") else 0)
    if kind == "linear":
        return {"bytes": elements * es + n * cols * _MX4_BYTES + rows * n * es, "flops": 2 * elements * n}
    if kind == "grad":
        return {"bytes": rows * n * es + (n * cols + elements) * _MX4_BYTES + elements * es + n * cols * 4, "flops": 4 * elements * n}
    if kind == "trip":
        return {"bytes": elements * (es + (1 + case["both"]) * (_MX4_BYTES + es)), "flops": elements * (1 + case["both"]) * 10}
    if kind == "norm":
        return {"bytes": 4 * elements * es + 2 * cols * es + gate + 8 * rows, "flops": 10 * elements}
    if kind == "entry":
        return {"bytes": 3 * elements * es + 2 * cols * es + gate + n * cols * _MX4_BYTES + rows * n * es,
                "flops": (20 + 2 * n) * elements}
    return {"bytes": 6 * elements * es + 2 * cols * (es + 4) + gate * (1 + 4 // es) + 8 * rows, "flops": 24 * elements}


# ---------------------------------------------------------------- the definitions in 64 bits

def _rotation():
    h2 = torch.tensor([[1.0, 1.0], [1.0, -1.0]], dtype=torch.float64, device="cuda")
    m = h2
    for _ in range(4):
        m = torch.kron(h2, m)
    return m / math.sqrt(32)


def _exact_mx4(x, transform, cover):
    """Values of the mx4 form in 64 bits, rotated blocks left rotated, from the grid's spacing."""
    y = torch.nn.functional.pad(x, (0, -x.shape[1] % 32)).view(-1, 32)
    if transform:
        y = torch.mm(y, _rotation())
    top = y.abs().max(1, keepdim=True).values
    mantissa, exponent = torch.frexp(top)                        # top = mantissa * 2^exponent, mantissa in [1/2, 1)
    e = exponent.to(torch.float64) - 3
    if cover:
        e = e + (mantissa > 0.75)
    scale = torch.exp2(torch.where(top > 0, e, 0.0).clamp_min(-127))
    a = (y / scale).abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(torch.float64)
    a = (torch.round(a / step) * step).clamp_max(6)
    return (torch.where(y < 0, -a, a) * scale).view(x.shape[0], -1)


def _exact_norm(s):
    c = s["case"]
    b, r = s["block"].double(), s["residual"].double()
    rb = 1 / torch.sqrt((b * b).sum(1) / c["cols"] + _EPS)
    p = b * rb[:, None] * s["w_post"].double()
    if s["gate"] is not None:
        p *= s["gate"].double()[torch.arange(c["rows"], device="cuda") // c["gate_rows"]]
    out = _RESIDUAL_SCALE * r + p
    rr = 1 / torch.sqrt((out * out).sum(1) / c["cols"] + _EPS)
    return out, out * rr[:, None] * s["w_pre"].double(), torch.stack((rb, rr))


def exact(case, seed):
    s = _inputs(case, seed)
    kind, options = case["kind"], (case.get("transform"), case.get("cover"))
    if kind == "linear":
        return torch.mm(_exact_mx4(s["x"].double(), *options), _exact_mx4(s["weight"].double(), *options).t())
    if kind == "grad":
        dy = s["grad_y"].double()
        w, x = (_exact_mx4(s[k].double().t().contiguous(), *options) for k in ("weight", "x"))
        return {"grad_x": torch.mm(_exact_mx4(dy, *options), w.t()),
                "grad_w": torch.mm(_exact_mx4(dy.t().contiguous(), *options), x.t())}
    if kind == "trip":
        got = []
        for x in (s["x"], s["x"].t())[:1 + case["both"]]:
            v = _exact_mx4(x.double().contiguous(), *options)
            if case["transform"]:
                v = torch.mm(v.view(-1, 32), _rotation()).view(v.shape)
            got.append(v[:, :x.shape[1]])
        return tuple(got)
    if kind == "norm":
        out, h, stats = _exact_norm(s)
        return {"residual": out, "h": h, "stats": stats}
    if kind == "entry":
        out, h, _ = _exact_norm(s)
        return {"residual": out, "y": torch.mm(_exact_mx4(h, *options), _exact_mx4(s["weight"].double(), *options).t())}
    # normgrad: the norms' Jacobians, symmetric, applied to what comes back
    rows, cols, stats = case["rows"], case["cols"], s["stats"].double()

    def back(u, unit, rstd):
        return (u - unit * ((u * unit).sum(1, keepdim=True) / cols)) * rstd[:, None]

    unit_b, unit_r = s["block"].double() * stats[0][:, None], s["residual_out"].double() * stats[1][:, None]
    total = s["grad_residual_out"].double() + back(s["grad_h"].double() * s["w_pre"].double(), unit_r, stats[1])
    out = {"grad_residual": _RESIDUAL_SCALE * total, "grad_w_pre": (s["grad_h"].double() * unit_r).sum(0)}
    through = total
    if s["gate"] is not None:
        group = torch.arange(rows, device="cuda") // case["gate_rows"]
        one_hot = (group[None] == torch.arange(s["gate"].shape[0], device="cuda")[:, None]).double()
        out["grad_gate"] = torch.mm(one_hot, total * unit_b * s["w_post"].double())
        through = total * s["gate"].double()[group]
    out["grad_w_post"] = (through * unit_b).sum(0)
    out["grad_block"] = back(through * s["w_post"].double(), unit_b, stats[0])
    return out
