"""Heads of prompts: more groups of heads to a token than one, several tokens to a wavefront, keys behind queries within a group, against the 64-bit definition, with the bounds of
test_gpu_heads.py; and which way through tokens and groups each shape takes."""
import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from oracle import heads64
from test_gpu_heads import EPS, HALF, KINDS, UNIT, _frequencies, _make, _values

pytestmark = pytest.mark.gpu

WAVES = 4
# tokens, query heads, key heads, channels, rotated.  Tokens split among wavefronts (below 1024), group by group, with more groups than wavefronts at work; and not split: several groups to
# a token, several tokens to a wavefront one after another.  Chunks of 16, 8 and 4 bytes and numbers one by one (halves of odd size).
SHAPES = [(1000, 40, 8, 128, 128), (1023, 17, 5, 128, 64), (1024, 13, 6, 128, 128), (4100, 13, 3, 128, 128), (6500, 9, 9, 64, 64), (3300, 19, 2, 96, 48), (1500, 21, 11, 58, 58), (5300, 9, 10, 50, 50),
          (5200, 17, 3, 36, 36), (2100, 7, 3, 256, 128)]


def _chunk(head, rotated, kind, pairs):
    """As in csrc/tahq_heads.hip: elements of a chunk, lanes to a head."""
    chunk = 16 // (2 if kind == "bf16" else 4)
    while chunk > 1 and not (head % chunk == 0 and rotated % (chunk if pairs else 2 * chunk) == 0 and head <= 128 * chunk):
        chunk //= 2
    need = (-(-head // chunk) + 1) // 2 if chunk > 1 else -(-(-(-head // 2)) // 4)
    lanes = 1
    while lanes < need:
        lanes *= 2
    return chunk, lanes


def _ways():
    """(shape, type, layout, chunk, groups to a token forward, groups of queries backward, whether a backward pass with norms has more work than wavefronts are at work at once, whether
    queries end within a group)."""
    for shape in SHAPES:
        tokens, hq, hk, head, rotated = shape
        for kind in KINDS:
            for pairs in (0, 1):
                chunk, lanes = _chunk(head, rotated, kind, pairs)
                each = 64 // lanes
                per_cu = 3 if chunk == 8 else 4 if chunk == 1 or (kind == "f32" and chunk == 4 and pairs) else 5
                work = sum(-(-tokens // max(each // n, 1)) * (-(-n // each) if tokens < 1024 else 1) for n in (hq, hk))
                yield shape, kind, pairs, chunk, -(-(hq + hk) // each), -(-hq // each), work > 256 * per_cu * WAVES, hq % each != 0


def test_shapes_go_every_way():
    """Several groups to a token of one wavefront, and several tokens to it, in every kind of chunk; keys in the group of the last queries; more groups than wavefronts, too, where a token's
    are shared."""
    ways = list(_ways())
    prompts = [w for w in ways if w[0][0] >= 1024]
    for kind, chunks in (("f32", {1, 2, 4}), ("bf16", {1, 2, 4, 8})):
        assert {w[3] for w in prompts if w[1] == kind and w[4] > 1} == chunks
        assert {w[3] for w in prompts if w[1] == kind and w[5] > 1 and w[6]} == chunks
    assert any(w[7] and w[4] > 1 for w in prompts) and any(w[6] and w[4] > 1 for w in ways if w[0][0] < 1024)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("pairs", (0, 1))
@pytest.mark.parametrize("norm", (1, 0))
def test_prompts(shape, kind, pairs, norm):
    tokens, hq, hk, head, rotated = shape
    t = _make(shape, kind, seed=tokens)
    t["positions"] = torch.arange(tokens) % 777 + 5      # samples one after another: another angle for every token
    table, f = _frequencies(rotated, "plain", 1.0)
    ld = (hq + 2 * hk) * head
    cfg = tahq.make_heads_config(tokens, hq, hk, head, rotated, KINDS[kind][0], layout=pairs, norm=norm, eps=EPS, ldq=ld, ldk=ld)
    packed = torch.cat((t["q"].flatten(1), t["k"].flatten(1), torch.zeros(tokens, hk * head, dtype=t["q"].dtype)), 1).cuda()
    views = lambda v: (v[:, :hq * head].unflatten(1, (hq, head)), v[:, hq * head:(hq + hk) * head].unflatten(1, (hk, head)))      # noqa: E731
    w = [t["w_" + n].cuda() if norm else None for n in "qk"]
    positions, grads = t["positions"].cuda(), [t["grad_" + n].cuda() for n in "qk"]
    heads = tahq.HeadRotary(cfg, tahq.make_rotary_config(rotated))
    out = heads.forward(*views(packed), *w, positions)
    place = torch.full((tokens, ld), 7.0, dtype=packed.dtype, device="cuda")
    got = heads.backward(*grads, *views(packed), *w, positions, out=views(place))
    torch.cuda.synchronize()
    assert (place[:, (hq + hk) * head:] == 7).all()
    p = t["positions"].numpy()
    for n, y, count in (("q", out[0], hq), ("k", out[1], hk)):
        weight = _values(t["w_" + n]) if norm else None
        want, size = heads64.forward(_values(t[n]), weight, p, f, rotated, pairs, EPS, 1.0)
        assert (np.abs(_values(y) - want) <= 32 * UNIT * size + HALF[kind] * np.abs(want) + 1e-38).all(), n
        want, size, dw, dw_size = heads64.backward(_values(t["grad_" + n]), _values(t[n]), weight, p, f, rotated, pairs, EPS, 1.0)
        assert (np.abs(_values(got["grad_" + n]) - want) <= 64 * UNIT * size + HALF[kind] * np.abs(want) + 1e-38).all(), n
        if norm:
            # a lane's sum over its tokens and groups, then trees: an eighth of the terms one after another at the most
            assert (np.abs(_values(got["grad_w_" + n]) - dw) <= (64 + tokens * count / 8) * UNIT * dw_size + 1e-38).all()


@pytest.mark.parametrize("shape", SHAPES[::3])
@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_in_place(shape, kind):
    """Outputs over queries and keys, gradients over the outputs' and over queries and keys: the same bits."""
    tokens, hq, hk, head, rotated = shape
    t = {n: v.cuda() for n, v in _make(shape, kind).items()}
    heads = tahq.HeadRotary(tahq.make_heads_config(*shape, KINDS[kind][0], eps=EPS), tahq.make_rotary_config(rotated))
    rest = (t["w_q"], t["w_k"], t["positions"])
    out = [v.clone() for v in heads.forward(t["q"], t["k"], *rest)]
    want = {n: v.clone() for n, v in heads.backward(t["grad_q"], t["grad_k"], t["q"], t["k"], *rest).items()}
    q, k = t["q"].clone(), t["k"].clone()
    heads.forward(q, k, *rest, out=(q, k))
    assert torch.equal(q, out[0]) and torch.equal(k, out[1])
    for over in ("grad_", ""):
        a = {n: t[n].clone() for n in ("grad_q", "grad_k", "q", "k")}
        got = heads.backward(a["grad_q"], a["grad_k"], a["q"], a["k"], *rest, out=(a[over + "q"], a[over + "k"]))
        assert all(torch.equal(got[n], want[n]) for n in want)
