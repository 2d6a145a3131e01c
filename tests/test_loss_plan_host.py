"""The plan of a loss over a vocabulary (csrc/tahq_loss_plan.hpp), compiled for the host: pieces, kinds of tiles, shares, places in the workspace."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2506_01352_amd as tahq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "tahq_loss_plan.hpp"
extern "C" void plan(const tahq_loss_config *c, int backward, uint64_t *out)
{
    const tahq::LossPlan p = tahq::plan_loss(c, backward != 0);
    const uint64_t v[] = {p.planes, p.copy, p.few, p.split, p.es, p.whole, p.blocks, p.padded, p.piece, (uint64_t)p.kind, (uint64_t)p.x_kind, p.parts, p.x_stages, p.x_slots, p.x_groups, p.x_plane,
                          p.g_plane, p.rows, p.targets, p.counts, p.x, p.at_target, p.running, p.stats, p.grads, p.sums, p.weight, p.total};
    for (unsigned i = 0; i < sizeof v / sizeof *v; ++i) out[i] = v[i];
}
extern "C" void shares(uint32_t tiles, uint32_t first, uint32_t stages, uint32_t slots, uint32_t *out)
{
    const tahq::Shares s(tiles, first, stages, slots);
    out[0] = s.parts;
    out[1] = s.run;
}
"""
NAMES = ("planes copy few split es whole blocks padded piece kind x_kind parts x_stages x_slots x_groups x_plane g_plane rows targets counts x at_target running stats grads sums "
         "weight total").split()
TILES = {0: (256, 256), 1: (128, 128), 2: (32, 128)}


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    (where / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_01352_amd", "csrc"),
                    str(where / "plan.cpp"), "-o", str(where / "plan.so")], check=True)
    return C.CDLL(str(where / "plan.so"))


@pytest.fixture(scope="module")
def plan(library):
    def run(backward, *sizes, **more):
        cfg, out = tahq.make_loss_config(*sizes, **more), (C.c_uint64 * len(NAMES))()
        library.plan(C.byref(cfg), backward, out)
        return dict(zip(NAMES, out))
    return run


SIZES = [(1, 1, 1), (5, 1600, 50257), (333, 1001, 32003), (2048, 1600, 50257), (8192, 4096, 131072), (65536, 8, 70001), (4100, 4100, 70), (1 << 23, 64, 1000), (1, 8, (1 << 31) - 1),
         (1 << 20, 65536, 1 << 30), (40, 33, 1 << 28)]


@pytest.mark.parametrize("rows, cols, vocab", SIZES)
@pytest.mark.parametrize("dtype", (tahq.F32, tahq.BF16))
@pytest.mark.parametrize("backward", (0, 1))
def test_places_hold_what_they_are_for(plan, rows, cols, vocab, dtype, backward):
    p = plan(backward, rows, cols, vocab, dtype)
    n = 3 if p["planes"] else 1
    assert p["es"] == (4 if dtype == tahq.F32 and not p["planes"] else 2) and p["whole"] * p["es"] == 64 and not (p["planes"] and dtype == tahq.BF16)
    assert p["blocks"] == -(-cols // p["whole"]) and rows <= p["padded"] < rows + p["whole"] and p["padded"] % p["whole"] == 0
    assert p["few"] == (not backward and rows <= 32 and (cols % p["whole"] != 0 or vocab <= 8192)) and p["copy"] == (not p["few"] and (cols % p["whole"] != 0 or p["planes"]))
    x_plane = p["padded"] * p["blocks"] * 64
    places = [("rows", 4 * p["padded"]), ("targets", 4 * p["padded"]), ("counts", 4 * -(-rows // 4096)), ("x", n * x_plane)]
    widest = min(vocab, p["piece"])
    if backward:
        tile = TILES[p["x_kind"]]
        stages = -(-widest // p["whole"])
        assert p["x_groups"] == max(-(-rows // tile[0]) * -(-cols // tile[1]), p["x_slots"]) and p["x_stages"] == stages and p["g_plane"] == p["padded"] * stages * 64
        places += [("grads", n * p["g_plane"]), ("sums", p["x_groups"] * tile[0] * tile[1] * 4)]
    else:
        tn, along = TILES[p["kind"]][1], 4 if p["kind"] == 2 else 2
        assert p["parts"] >= -(-widest // tn) * along
        places += [("at_target", 4 * p["padded"]), ("running", 8 * p["padded"]), ("stats", 8 * p["padded"] * p["parts"])]
    places += [("weight", n * -(-widest // p["whole"]) * p["whole"] * p["blocks"] * 64 if p["copy"] else 0)]
    at = 256
    for name, size in places:
        assert p[name] % 256 == 0 and p[name] >= at, name
        at = p[name] + size
    assert at <= p["total"] and p["x_plane"] == x_plane


@pytest.mark.parametrize("rows, cols, vocab", SIZES)
@pytest.mark.parametrize("dtype", (tahq.F32, tahq.BF16))
@pytest.mark.parametrize("backward", (0, 1))
def test_offsets_fit_32_bits(plan, rows, cols, vocab, dtype, backward):
    """What a lane adds to a uniform address: blocks of a tile (eight at the most) times a block's bytes, and rows of a tile times a row's bytes."""
    p = plan(backward, rows, cols, vocab, dtype)
    assert p["piece"] % 256 == 0 and p["piece"] <= 1 << 22
    for block_rows in (p["padded"], p["piece"]):
        assert 7 * block_rows * 64 + 2048 < 1 << 32
    assert 256 * cols * (4 if dtype == tahq.F32 else 2) < 1 << 32


def test_later_pieces_have_no_more_parts_than_the_first(library):
    """Parts cover a piece's stages, each has one at least, and a later piece, which is no longer, adds to parts that the first one has written."""
    out = (C.c_uint32 * 2)()

    def shares(*a):
        library.shares(*a, out)
        return out[0], out[1]

    for tiles in (0, 1, 2, 3, 4, 5, 7, 9, 16, 33, 100, 511, 512, 513, 5000):
        for first in (1, 8, 15, 16, 17, 31, 129, 250, 480, 485, 490, 2048, 7704, 8192, 8200):
            parts, run = shares(tiles, first, first, 512)
            assert (parts - 1) * run < first <= parts * run and (parts == 1 or (run >= 16 and parts * tiles <= 512))
            for stages in {1, 2, 15, 16, 17, first // 3 + 1, first // 2 + 1, 480, 2048, first}:
                if stages <= first:
                    later, each = shares(tiles, first, stages, 512)
                    assert later <= parts and (later - 1) * each < stages <= later * each


def test_which_tiles_the_gpu_tests_take(plan):
    """The sizes of the GPU tests, so that other constants do not take a kind of tile, or fp32 in planes, out of them: tiles of logits forward and
    backward, and of the hidden states' gradient."""
    def kinds(*s, dtype=tahq.BF16):
        f, b = plan(0, *s, dtype), plan(1, *s, dtype)
        return f["kind"], b["kind"], b["x_kind"]

    assert kinds(5, 32, 127) == (2, 2, 2) and kinds(130, 1600, 257) == (1, 1, 1) and kinds(500, 40, 32601) == kinds(500, 96, 32601) == (0, 0, 1) and kinds(257, 512, 9000)[2] == 1
    assert kinds(1030, 2056, 4099)[2] == kinds(1030, 2080, 4099)[2] == 0 and kinds(2048, 1600, 50257) == (0, 0, 0)
    few = [(plan(0, *s, dtype)["few"], plan(0, *s, dtype)["split"]) for s in ((5, 1600, 8192), (7, 1001, 700), (5, 1001, 9001), (20, 384, 9001)) for dtype in (tahq.F32, tahq.BF16)]
    assert few == [(1, 1)] * 4 + [(1, 0)] * 2 + [(0, 0)] * 2
    assert plan(1, 4100, 40, 40001, tahq.BF16)["piece"] < 40001 and plan(0, 65536, 8, 70001, tahq.BF16)["piece"] < 70001
    assert plan(0, 300, 64, 5003, tahq.F32)["copy"] == 0 and plan(0, 300, 40, 33003, tahq.BF16)["copy"] == 1
    planes = [(plan(0, *s, tahq.F32)["planes"], plan(1, *s, tahq.F32)["planes"]) for s in ((130, 1600, 257), (300, 64, 11003), (1030, 260, 4099), (161, 31, 17000), (161, 31, 300))]
    assert planes == [(0, 0), (0, 1), (1, 1), (1, 1), (0, 0)]
    f32 = lambda *s: kinds(*s, dtype=tahq.F32)      # noqa: E731
    assert f32(200, 64, 16001) == f32(100, 33, 32001) == (1, 1, 1) and f32(66, 260, 4099)[:2] == f32(130, 1600, 257)[:2] == f32(64, 257, 1000)[:2] == (2, 2)
    assert f32(1030, 260, 4099) == (1, 1, 1) and f32(700, 64, 33003)[:2] == (0, 0) and f32(1030, 2056, 4099)[2] == 0 and f32(300, 4104, 4200)[2] == 1
