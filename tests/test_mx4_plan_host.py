"""How products are cut (csrc/tahq_mx4_plan.hpp), compiled for the host (CPU): every kind of tile is what some tested shape gets."""
import os
import subprocess

import pytest

from mx4_products import FEW, PRODUCTS, T64_TEAMS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include <cstdio>
#include "tahq_mx4_plan.hpp"

int main()
{
    tahq_mx4_matmul_config c = {};
    while (std::scanf("%u %u %u %u", &c.m, &c.n, &c.k, &c.out_dtype) == 4) {
        const tahq::ProductPlan p = tahq::plan_product(&c);
        std::printf("%d %u %u %llu\n", p.kind, p.run, p.parts, (unsigned long long)tahq::product_workspace(&c));
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    source, program = where / "plan.cpp", where / "plan"
    source.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-ffp-contract=off", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2506_01352_amd", "csrc"), str(source), "-o", str(program)], check=True)

    def run(shapes):
        text = "\n".join(f"{m} {n} {k} {1 if kind == 'bf16' else 0}" for m, n, k, kind in shapes)
        out = subprocess.run([str(program)], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return run


def test_tested_products_are_cut_as_they_say(plan):
    got = plan([(m, n, k, c) for _, _, c, m, n, k in PRODUCTS])
    for (kind, parts, _, m, n, k), (of, run, pieces, ws) in zip(PRODUCTS, got):
        assert (of, pieces > 1) == (kind, parts), (m, n, k, of, pieces)
        assert run * (pieces - 1) < -(-k // 256) <= run * pieces and ws == (pieces * m * n * 4 if pieces > 1 else 0)


def test_every_kind_is_tested_in_both_types_and_every_round_of_buffers():
    kinds = {(kind, parts, c) for kind, parts, c, *_ in PRODUCTS}
    assert kinds == {(k, False, c) for k in range(FEW, T64_TEAMS + 1) for c in ("bf16", "f32")} | {(4, True, c) for c in ("bf16", "f32")}
    for kind, rounds in ((0, 2), (1, 3), (2, 2)):
        assert {-(-k // 256) % rounds for of, _, _, _, _, k in PRODUCTS if of == kind} == set(range(rounds))
