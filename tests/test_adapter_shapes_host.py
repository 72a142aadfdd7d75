"""The launch shapes of the adapters' kernels (apb_adapter_shape.h), compiled with the host compiler: the sizes that the GPU tests take
reach every form of every kernel, and the slices of a gradient have places of their own."""
import os
import subprocess

import numpy as np
import pytest

import adapter_cases as cases

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ASK = r"""
#include <cstdio>
#include "apb_adapter_shape.h"
using namespace apb;

int main() {
    char what;
    int S, L, M, K, r;
    while (std::scanf(" %c %d %d %d %d %d", &what, &S, &L, &M, &K, &r) == 6) {
        const DownPlan p = down_plan(S, M, K, r);
        if (what == 'd') std::printf("%d %d %d %d %d\n", p.rt, p.jt, p.parts, down_waves(p.rt, p.jt), p.tile);
        else if (what == 'u') std::printf("%d\n", up_rows(S, M, K));
        else if (what == 'g' || what == 'w') {                        // (w: an X of float32)
            const GradientForm f = gradient_form_of(what == 'w' ? APB_F32 : APB_BF16, S, L, M, K, r);
            std::printf("%d %d %d %d %d\n", gradient_rows(S, L, M, K, r), f.jt, f.nc, f.waves, gradient_by_segment(S, L, K, r));
        }
        else std::printf("%d %lld\n", place_of_slices(S, L), places_of_slices(M, L));      // (S: rows before, L: rows to a slice)
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


def _sizes():
    """(segments, adapters, rows, long side, rank) of every call that the GPU test makes of each case."""
    for M, K, N, r, L, kind in cases.CASES:
        off, _ = cases.segments(kind, M, L, r)
        S = 1 if off is None else len(off) - 1
        for side in (K, N):
            yield S, L, M, side, r


def test_cases_reach_every_form(ask):
    sizes = list(_sizes())
    down = ask([("d", *s) for s in sizes])
    assert {d[:2] for d in down} == {(rt, jt) for rt in (1, 2, 4) for jt in (1, 2, 4)}
    assert {d[2] for d in down} >= {1, 2, 4, 8}
    assert {(d[0], d[4] < 16 * d[0]) for d in down} == {(1, False), (2, False), (2, True), (4, False), (4, True)}
    # the kernel that streams rows past B, by ranks held (16, 32, 64, 128; above, and in float32, the other one), rows and width
    up = ask([("u", *s) for s in sizes])
    held = lambda r: 0 if r <= 16 else 1 if r <= 32 else 2 if r <= 64 else 4 if r <= 128 else None
    reached = {(held(s[4]), rows[0] > 16) for s, rows in zip(sizes, up)}
    assert reached == {(h, many) for h in (0, 1, 2, 4, None) for many in (False, True)}
    assert {rows[0] for rows in up} == {16, 32, 64}
    assert {(s[3] % 128 == 0, s[3] < 8, s[3] < 128) for s in sizes} == {(True, False, False), (False, False, False), (False, True, True), (False, False, True)}
    grad, wide = ask([("g", *s) for s in sizes]), ask([("w", *s) for s in sizes])
    assert {g[1:4] for g in grad} == {(j, 4, w) for j in (1, 2, 4) for w in (1, 4, 8)} | {(j, 8, 8) for j in (1, 2)}
    assert {g[1:4] for g in wide} == {(j, 4, w) for j in (1, 2, 4) for w in (1, 4, 8) if (j, w) != (4, 8)}
    assert {(g[1], g[3], s[3] < 64) for s, g in zip(sizes, grad)} == {(j, w, tiny) for j in (1, 2, 4) for w in (1, 4, 8) for tiny in (False, True)}
    assert {(g[1], s[2] > g[0]) for s, g in zip(sizes, grad)} == {(j, shared) for j in (1, 2, 4) for shared in (False, True)}
    assert {(g[4], s[2] > g[0]) for s, g in zip(sizes, grad)} == {(b, shared) for b in (0, 1) for shared in (False, True)}
    assert any(s[2] > g[0] and g[2] == 8 for s, g in zip(sizes, grad))
    assert any(s[3] % 128 and g[2] == 8 for s, g in zip(sizes, grad))
    assert any(s[2] > 1024 and s[1] == 1 for s in sizes)             # (more rows of one adapter than a list holds, without a workspace)


def test_slices_have_places_of_their_own(ask):
    g = np.random.default_rng(0)
    for _ in range(200):
        L, each = int(g.integers(1, 30)), int(g.choice([1, 2, 3, 64, 128, 320]))
        rows = np.where(g.random(L) < 0.3, 0, np.exp(g.uniform(0, 8, L))).astype(int)
        if g.random() < 0.3:
            rows[g.integers(L)] = each + 1
        before, M = np.concatenate([[0], np.cumsum(rows)[:-1]]), max(int(rows.sum()), 1)
        first = ask([("p", int(b), each, M, 1, 1) for b in before])
        taken = [p + z for (p, _), n in zip(first, rows) if n > each for z in range(-(-int(n) // each))]
        assert len(set(taken)) == len(taken)
        assert not taken or max(taken) < first[0][1]


def test_plans_over_the_range(ask):
    """What every size has to keep: parts that are whole lines of K, a workspace that is a size, groups that a kernel exists for."""
    g = np.random.default_rng(1)
    sizes = [(int(np.exp(g.uniform(0, 8.3))), int(np.exp(g.uniform(0, 8.3))), int(np.exp(g.uniform(0, 16.6))), int(np.exp(g.uniform(0, 15.2))),
              int(g.integers(1, 257))) for _ in range(2000)] + [(4096, 4096, 1 << 24, 1 << 22, 256), (1, 1, 1, 1, 1)]
    for (rt, jt, parts, waves, tile), (S, L, M, K, r) in zip(ask([("d", *s) for s in sizes]), sizes):
        assert rt in (1, 2, 4) and jt in (1, 2, 4) and 1 <= parts <= 8 and (parts == 1 or K >= 512 * parts)
        assert tile == 16 if rt == 1 else 8 * rt < tile <= 16 * rt
        assert waves * 2 * (rt + jt) * 1024 <= 160 * 1024 and waves * rt * jt * 1024 <= 160 * 1024      # (LDS)
    for what in "gw":
        for (each, jt, nc, waves, by_segment), (S, L, M, K, r) in zip(ask([(what, *s) for s in sizes]), sizes):
            assert 256 <= each and -(-M // each) <= 65535 and 2 * M // each < 1 << 31 and L * -(-r // (16 * jt)) <= 65535
            assert waves * jt * nc * 1024 + (1024 + 32) * 4 <= 160 * 1024      # (LDS)
            assert nc == 4 or K >= 128                                         # (no form for fewer columns)
