"""The plan of a loss over a vocabulary (csrc/tahq_loss_plan.hpp), compiled for the host: pieces, kinds of tiles, places in the workspace."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2506_01352_amd as tahq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "tahq_loss_plan.hpp"
extern "C" void plan(const tahq_loss_config *c, uint64_t *out)
{
    const tahq::LossPlan p = tahq::plan_loss(c);
    const uint64_t v[] = {p.forward_piece, p.backward_piece, (uint64_t)p.forward_kind, (uint64_t)p.grads_kind, (uint64_t)p.x_kind, p.parts, p.x_slots, p.x_groups, p.padded, p.ldx,
                          p.pad, p.rows, p.targets, p.counts, p.x, p.at_target, p.running, p.stats, p.forward_weight, p.forward_total, p.grads, p.sums, p.backward_weight,
                          p.backward_total, p.whole, p.x_stages};
    for (unsigned i = 0; i < sizeof v / sizeof *v; ++i) out[i] = v[i];
}
"""
NAMES = ("forward_piece backward_piece forward_kind grads_kind x_kind parts x_slots x_groups padded ldx pad rows targets counts x at_target running stats "
         "forward_weight forward_total grads sums backward_weight backward_total whole x_stages").split()
TILES = {0: (256, 256), 1: (128, 128), 2: (32, 128)}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    (where / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_01352_amd", "csrc"),
                    str(where / "plan.cpp"), "-o", str(where / "plan.so")], check=True)
    lib = C.CDLL(str(where / "plan.so"))

    def run(*sizes, **more):
        cfg, out = tahq.make_loss_config(*sizes, **more), (C.c_uint64 * len(NAMES))()
        lib.plan(C.byref(cfg), out)
        return dict(zip(NAMES, out))
    return run


SIZES = [(1, 1, 1), (5, 1600, 50257), (333, 1001, 32003), (2048, 1600, 50257), (8192, 4096, 131072), (65536, 8, 70001), (4100, 4100, 70), (1 << 23, 64, 1000), (1, 8, (1 << 31) - 1),
         (1 << 20, 65536, 1 << 30), (40, 33, 1 << 28)]


@pytest.mark.parametrize("rows, cols, vocab", SIZES)
@pytest.mark.parametrize("dtype", (tahq.F32, tahq.BF16))
def test_places_hold_what_they_are_for(plan, rows, cols, vocab, dtype):
    p, es = plan(rows, cols, vocab, dtype), 4 if dtype == tahq.F32 else 2
    assert p["ldx"] % p["whole"] == 0 and cols <= p["ldx"] < cols + p["whole"] and p["pad"] == (p["ldx"] != cols) and rows <= p["padded"] < rows + p["whole"]
    common = [("rows", 4 * p["padded"]), ("targets", 4 * p["padded"]), ("counts", 4 * -(-rows // 4096)), ("x", p["padded"] * p["ldx"] * es)]
    tn, along = TILES[p["forward_kind"]][1], 4 if p["forward_kind"] == 2 else 2
    assert p["parts"] >= min(-(-vocab // tn), p["forward_piece"] // tn) * along
    forward = common + [("at_target", 4 * p["padded"]), ("running", 8 * p["padded"]), ("stats", 8 * p["padded"] * p["parts"]),
                        ("forward_weight", min(p["forward_piece"], -(-vocab // p["whole"]) * p["whole"]) * p["ldx"] * es if p["pad"] else 0)]
    widest = min(vocab, p["backward_piece"])
    tile = TILES[p["x_kind"]]
    tiles = -(-rows // tile[0]) * -(-cols // tile[1])
    assert p["x_groups"] == max(tiles, p["x_slots"]) and p["x_stages"] == -(-widest // p["whole"])
    backward = common + [("grads", p["padded"] * -(-widest // p["whole"]) * 64), ("sums", p["x_groups"] * tile[0] * tile[1] * 4),
                         ("backward_weight", -(-widest // p["whole"]) * 64 * p["ldx"] // p["whole"] * p["whole"] if p["pad"] else 0)]
    for places, total in ((forward, p["forward_total"]), (backward, p["backward_total"])):
        at = 256
        for name, size in places:
            assert p[name] % 256 == 0 and p[name] >= at, name
            at = p[name] + size
        assert at <= total


@pytest.mark.parametrize("rows, cols, vocab", SIZES)
@pytest.mark.parametrize("dtype", (tahq.F32, tahq.BF16))
def test_offsets_fit_32_bits(plan, rows, cols, vocab, dtype):
    """What a lane adds to a uniform address: blocks of a tile (eight at the most) times a block's bytes, and rows of a tile times a row's bytes."""
    p, es = plan(rows, cols, vocab, dtype), 4 if dtype == tahq.F32 else 2
    assert p["forward_piece"] % 256 == 0 and p["backward_piece"] % 256 == 0 and max(p["forward_piece"], p["backward_piece"]) <= 1 << 22
    for block_rows in (p["padded"], p["backward_piece"]):
        assert 7 * block_rows * 64 + 2048 < 1 << 32
    assert 256 * cols * es < 1 << 32


def test_which_tiles_the_gpu_tests_take(plan):
    """The sizes of the GPU tests, so that other constants do not take a kind of tile out of them: (forward, gradients of logits, of hidden states)."""
    kinds = lambda *s: tuple(plan(*s, tahq.BF16)[k] for k in ("forward_kind", "grads_kind", "x_kind"))      # noqa: E731
    assert kinds(5, 32, 127) == (2, 2, 2) and kinds(130, 1600, 257) == (1, 1, 1) and kinds(300, 40, 33003) == (0, 0, 1) and kinds(257, 512, 9000)[2] == 1
    assert kinds(1030, 2056, 4099)[2] == 0 and kinds(2048, 1600, 50257) == (0, 0, 0)
    assert plan(4100, 40, 40001, tahq.BF16)["backward_piece"] < 40001 and plan(65536, 8, 70001, tahq.BF16)["forward_piece"] < 70001
    assert plan(300, 64, 5003, tahq.F32)["pad"] == 0 and plan(300, 40, 33003, tahq.BF16)["pad"] == 1
