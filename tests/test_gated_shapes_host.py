"""The tile rule of the gated products (apb_mx4_shape.h), compiled with the host compiler, and who takes the single kernel."""
import os
import subprocess

import pytest

import gated_cases as cases

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2306_08960_amd", "libapb.so")

ASK = r"""
#include <cstdio>
#include "apb_mx4_shape.h"

int main() {
    int M, N, E;
    while (std::scanf("%d %d %d", &M, &N, &E) == 3) std::printf("%d\n", apb::mx4_gated_side(M, N, E ? E : 1, E > 0));
}
"""


def test_cases_reach_every_tile_size(tmp_path):
    src, exe = tmp_path / "ask.cpp", tmp_path / "ask"
    src.write_text(ASK)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-ftrapv", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2306_08960_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    text = "\n".join(f"{M} {N} {E}" for M, N, _, E, _ in cases.PRODUCTS)
    p = subprocess.run([str(exe)], input=text, stdout=subprocess.PIPE, text=True, check=True, timeout=60)
    assert [int(v) for v in p.stdout.split()] == [side for *_, side in cases.PRODUCTS]
    for grouped in (False, True):
        assert {side for *_, E, side in cases.PRODUCTS if (E > 0) == grouped} == {64, 128, 256}


@pytest.mark.skipif(not os.path.exists(LIB), reason="libapb.so not built")
def test_cases_reach_both_kernels():
    from paper_2306_08960_amd import binding as b
    one = [b.apb_mx4_gated_linear_scratch_bytes(E > 0, max(E, 1), M, N, K) == 0 for M, N, K, E, _ in cases.PRODUCTS]
    assert {side for (*_, side), o in zip(cases.PRODUCTS, one) if not o} == {64, 128, 256}
    few = [c for c, o in zip(cases.PRODUCTS, one) if o]
    assert {(c[0] > 16, c[3] > 0) for c in few} >= {(False, False), (True, False), (True, True)}
    for M, N, K, E, _ in cases.PRODUCTS:
        assert b.apb_mx4_gated_linear_scratch_bytes(E > 0, max(E, 1), M, N, K, True) == b.apb_mx4_bytes(M, K)
