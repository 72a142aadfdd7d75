"""The tile rules of the 4-bit products and their gradients (apb_mx4_shape.h), compiled with the host compiler: the sizes that the GPU
tests take reach the kernels that they are there for."""
import os
import subprocess

import pytest

import mx4_tile_cases as cases

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPE = {"f32": 0, "bf16": 1, "f16": 2}

ASK = r"""
#include <cstdio>
#include "apb_mx4_shape.h"
using namespace apb;

int main() {
    char what;
    int type, E, M, N, K;
    while (std::scanf(" %c %d %d %d %d %d", &what, &type, &E, &M, &N, &K) == 6) {
        const bool grouped = E > 0;
        const int groups = grouped ? E : 1;
        if (what == 'y') {
            std::printf("%d\n", mx4_product_side(M, N));
        } else {
            const Mx4Plan p = what == 'x' ? mx4_gradient_plan<false>(type, grouped, groups, M, N, K)
                                          : mx4_gradient_plan<true>(type, grouped, groups, M, N, K);
            std::printf("%d %d %d\n", p.f, p.groups, p.slices);
        }
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    at = tmp_path_factory.mktemp("rules")
    src, exe = at / "ask.cpp", at / "ask"
    src.write_text(ASK)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-ftrapv", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2306_08960_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def answers(questions):
        text = "\n".join(" ".join(map(str, q)) for q in questions)
        p = subprocess.run([str(exe)], input=text, stdout=subprocess.PIPE, text=True, check=True, timeout=60)
        return [tuple(map(int, line.split())) for line in p.stdout.splitlines()]
    return answers


def test_products_reach_every_tile_size(ask):
    got = ask([("y", 0, E, M, N, K) for M, N, K, E, _ in cases.PRODUCTS])
    assert got == [(side,) for *_, side in cases.PRODUCTS]
    # (more than sixteen rows an expert: not the kernel for few rows)
    assert all(M > 16 * max(E, 1) for M, _, _, E, _ in cases.PRODUCTS)
    for plain in (True, False):
        assert {128, 256} <= {side for *_, E, side in cases.PRODUCTS if (E == 0) == plain}


def test_gradients_reach_every_kernel(ask):
    for i, what in ((5, "x"), (6, "w")):
        got = ask([(what, TYPE[t], E, M, N, K) for M, N, K, E, t, *_ in cases.GRADIENTS])
        assert got == [c[i] for c in cases.GRADIENTS]
        # what there is by type of the gradient: tiles of 256 and two groups of waves on one of 128 in bfloat16 alone; with and without
        # slices
        reached = {(c[4], *c[i][:2], c[i][2] > 1) for c in cases.GRADIENTS}
        assert reached >= {("bf16", 4, 1, False), ("bf16", 4, 1, True), ("bf16", 2, 2, False)}
        assert reached >= {(t, 2, 1, shared) for t in TYPE for shared in (False, True)}


def test_special_blocks_reach_every_tile_size(ask):
    for i, what in ((4, "x"), (5, "w")):
        assert ask([(what, TYPE[t], 0, M, N, K) for M, N, K, t, *_ in cases.SPECIAL]) == [c[i] for c in cases.SPECIAL]
        for f in (1, 2, 4):                                          # sums of whole passes and shorter ones
            long = {c[1 if what == "x" else 0] >= 64 for c in cases.SPECIAL if c[i][0] == f}
            assert long == {True, False}
