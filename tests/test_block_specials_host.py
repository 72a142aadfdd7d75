"""Gated blocks, 8-bit checkpoints and adapters without a GPU: NaN in the oracle, sizes at the limits, operands of another device."""
import ctypes
import os
import subprocess
import types

import numpy as np
import pytest
import torch

from oracle import block_oracle as o

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2306_08960_amd", "libapb.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libapb.so not built")


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
def test_nan_has_no_value_and_no_slope(kind):
    v, d, _, _ = o.act(np.array([np.nan, 1.0, -1.0]), kind)
    assert np.isnan(v[0]) and np.isnan(d[0]) and np.isfinite(v[1:]).all() and np.isfinite(d[1:]).all()


# ---- operands of another device: kernels are launched on the current one --------------------------------------------------

class _On(torch.Tensor):
    """Host memory that says it is on a GPU: nothing here gets as far as a launch."""
    where = 0
    is_cuda = True

    def get_device(self):
        return self.where


def _on(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_On)


def _operands():
    """Every entry point with every tensor it takes, by name, and its other arguments."""
    M, N, K, r, L, S = 40, 64, 96, 4, 2, 3
    bytes_, ints = (lambda n: _on(n, dtype=torch.uint8)), (lambda n: _on(n, dtype=torch.int32))
    mx4, mx8 = (lambda rows, k: bytes_(rows * (k + 255) // 256 * 136)), (lambda rows, k: bytes_(rows * (k + 31) // 32 * 33))
    seg = dict(offsets=ints(S + 1), adapter=ints(S))
    T = _on(1, M, r, dtype=torch.float32)
    return [
        ("apb_mx8_quantize", dict(X=_on(M, K), mx8=mx8(M, K)), {}),
        ("apb_mx8_dequantize", dict(mx8=mx8(M, K), X=_on(M, K)), dict(rows=M, K=K)),
        ("apb_mx4_gated_gemm", dict(A=mx4(M, K), W=mx4(2 * 2 * N, K), Y=_on(M, N), offsets=ints(3), saved=mx8(2 * M, N)), dict(M=M, N=N, K=K)),
        ("apb_mx4_gated_linear", dict(X=_on(M, K), W=mx4(2 * 2 * N, K), Y=_on(M, N), rows_from=ints(M), offsets=ints(3), scratch=mx4(M, K),
                                      saved=mx8(2 * M, N)), dict(N=N)),
        ("apb_gated_forward", dict(GU=_on(M, 2 * N), Y=_on(M, N), saved=mx8(2 * M, N)), {}),
        ("apb_gated_backward", dict(GU=_on(M, 2 * N), dY=_on(M, N), dGU=_on(M, 2 * N), Y=_on(M, N)), {}),
        ("apb_gated_backward", dict(GU=mx8(2 * M, N), dY=_on(M, N), dGU=_on(M, 2 * N), Y=_on(M, N)), {}),
        ("apb_adapter_down", dict(X=_on(M, K), A=_on(L, r, K), scale=_on(L, dtype=torch.float32), T=T, **seg), {}),
        ("apb_adapter_up", dict(T=T, B=_on(L, r, N), Y0=_on(M, N), Y=_on(M, N), **seg), {}),
        ("apb_adapter_gradient", dict(T=T, X=_on(M, K), dA=_on(L, r, K, dtype=torch.float32), workspace=bytes_(64), **seg), dict(L=L)),
        ("apb_adapter_gradient", dict(T=T, X=mx8(M, K), dA=_on(L, r, K, dtype=torch.float32), workspace=bytes_(64), **seg), dict(L=L, K=K)),
    ]


@needs_lib
@pytest.mark.parametrize("at", range(len(_operands())), ids=lambda i: f"{_operands()[i][0]}-{i}")
def test_no_operand_is_taken_from_another_device(monkeypatch, at):
    from paper_2306_08960_amd import binding
    real, launched = binding.load(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes") or name.endswith("_parts"):
                return getattr(real, name)
            return lambda *args: launched.append(name) or 0
    monkeypatch.setattr(binding, "load", Library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(binding, "_several_devices", True)
    name, tensors, sizes = _operands()[at]
    call = getattr(binding, name)
    call(**tensors, **sizes)
    call(**tensors, **sizes, stream=types.SimpleNamespace(cuda_stream=7, device_index=0))
    assert launched == [name] * 2
    for which in tensors:
        other = tensors[which].clone()
        other.where = 1
        with pytest.raises(ValueError, match="current device"):
            call(**{**tensors, which: other}, **sizes)
    with pytest.raises(ValueError, match="current device"):
        call(**tensors, **sizes, stream=types.SimpleNamespace(cuda_stream=7, device_index=1))
    assert launched == [name] * 2


# ---- sizes at the limits -------------------------------------------------------------------------------------------------------

P, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 1)     # never followed: the odd one is refused once the sizes are taken


@needs_lib
def test_limits_of_the_8_bit_form_hold_only_with_it():
    """2 M rows of N in 8 bits are bounded; a product that saves nothing takes what the plain 4-bit product takes."""
    from paper_2306_08960_amd import binding as b
    lib = b.load()
    gemm = lambda M, N, K, saved: lib.apb_mx4_gated_gemm(P, P, None, 1, M, N, K, 0, 1, ODD, N, saved, None)
    plain = lambda M, N, K: lib.apb_mx4_gemm(P, P, None, 1, M, N, K, 1, ODD, N, None)
    linear = lambda M, N, K, saved: lib.apb_mx4_gated_linear(P, 1, K, M, None, P, None, 1, M, N, K, 0, P, 1, ODD, N, saved, None)
    scratch = lambda M, N, K, saved: b.apb_mx4_gated_linear_scratch_bytes(False, 1, M, N, K, saved)
    M, N, K = 1 << 20, 16384, 4096                                   # 2 M * 512 blocks = 2^30
    assert plain(M, 2 * N, K) == b.APB_ERR_ALIGN
    assert gemm(M, N, K, None) == b.APB_ERR_ALIGN and gemm(M, N, K, P) == b.APB_ERR_SHAPE
    assert linear(M, N, K, None) == b.APB_ERR_ALIGN and linear(M, N, K, P) == b.APB_ERR_SHAPE
    assert scratch(M, N, K, False) == b.apb_mx4_bytes(M, K) > 0 and scratch(M, N, K, True) == 0
    most = ((1 << 30) - 64) // 512 // 2
    assert gemm(most, N, K, P) == b.APB_ERR_ALIGN and gemm(most + 1, N, K, P) == b.APB_ERR_SHAPE
    assert scratch(most, N, K, True) == b.apb_mx4_bytes(most, K) and scratch(most + 1, N, K, True) == 0
    N = 64 * 65535                                                   # (columns: 2 N is what the plain product takes at most)
    assert plain(1, 2 * N, 256) == b.APB_ERR_ALIGN and plain(1, 2 * N + 2, 256) == b.APB_ERR_SHAPE
    assert gemm(1, N, 256, None) == b.APB_ERR_ALIGN and gemm(1, N + 1, 256, None) == b.APB_ERR_SHAPE


@needs_lib
def test_limits_of_the_activation():
    """M rows of N, or 2 M where they are read from or written in 8 bits."""
    from paper_2306_08960_amd import binding as b
    lib = b.load()
    forward = lambda M, N, saved: lib.apb_gated_forward(P, 1, 2 * N, M, N, 0, ODD, N, saved, None)
    backward = lambda M, N, t: lib.apb_gated_backward(P, t, 2 * N, P, 1, N, M, N, 0, ODD, 2 * N, None, N, None)
    N, all_ = 32 * 512, ((1 << 30) - 64) // 512
    assert forward(all_, N, None) == b.APB_ERR_ALIGN and forward(all_ + 1, N, None) == b.APB_ERR_SHAPE
    assert forward(all_ // 2, N, P) == b.APB_ERR_ALIGN and forward(all_ // 2 + 1, N, P) == b.APB_ERR_SHAPE
    assert backward(all_, N, 1) == b.APB_ERR_ALIGN and backward(all_ + 1, N, 1) == b.APB_ERR_SHAPE
    assert backward(all_ // 2, N, 3) == b.APB_ERR_ALIGN and backward(all_ // 2 + 1, N, 3) == b.APB_ERR_SHAPE


@needs_lib
def test_limits_of_parts():
    from paper_2306_08960_amd import binding as b
    lib = b.load()
    up = lambda parts: lib.apb_adapter_up(P, parts, P, 1, P, P, 3, 2, 20, 64, 8, None, 64, ODD, 64, None)
    gradient = lambda parts: lib.apb_adapter_gradient(P, parts, P, 1, 64, P, P, 3, 2, 20, 64, 8, ODD, None, 0, None)
    for f in (up, gradient):
        assert f(8) == b.APB_ERR_ALIGN and f(9) == b.APB_ERR_SHAPE and f(0) == b.APB_ERR_SHAPE


@needs_lib
def test_little_work_is_bounded():
    """A product of less than 256 values a row costs what one of 256 does: how much runs as one kernel does not grow without end as there
    are fewer, and a launch of it is never more than a launch can be."""
    from paper_2306_08960_amd import binding as b
    one = lambda E, M, N, K: b.apb_mx4_gated_linear_scratch_bytes(E > 0, max(E, 1), M, N, K) == 0
    g = np.random.default_rng(0)
    taken = set()
    for _ in range(4000):
        E, M, N = int(g.choice([0, 16])), int(np.exp(g.uniform(3, 14))), int(np.exp(g.uniform(0, 11)))
        few = M <= 16 * max(E, 1) or (M * N >= 1 << 22 and M <= 32 * E if E else M <= 64 or M <= 256 and N > 24320)
        for K in (1, 8, 32, 100, 128, 255, 256):
            o = one(E, M, N, K)
            taken.add((E, K, few, o))
            assert o == few or not few
            if o and not few:
                assert M <= (16384 if E else 4096) and M * N <= 1 << (20 if E else 21) and M * N * K <= 1 << (27 if E else 28)
    assert {(E, K, o) for E, K, few, o in taken if not few} == {(E, K, o) for E in (0, 16) for K in (1, 8, 32, 100, 128, 255, 256) for o in (False, True)}
    for E, M, N, K in ((0, 4096, 2048, 32), (0, 1024, 8192, 8), (16, 131072, 4, 128), (16, 131072, 32, 32), (16, (1 << 27) - 8, 1, 1)):
        assert not one(E, M, N, K)
    for E, M, N, K in ((0, 4096, 256, 32), (16, 4096, 128, 32), (16, 16384, 32, 200), (0, 32, 262144, 8), (0, 64, 8192, 256), (0, 256, 24576, 32),
                       (16, 512, 8192, 32), (64, 2048, 16384, 256), (0, 310, 3664, 66), (9, 192, 4168, 160), (0, 1024, 512, 512)):
        assert one(E, M, N, K)


# ---- slices of the adapters' gradient: workgroups for those that there are ------------------------------------------------

SLICES = r"""
#include <cstdio>
#include "apb_adapter_shape.h"
using namespace apb;

int main() {
    char what;
    int a, b, c, K, r;
    while (std::scanf(" %c %d %d %d %d %d", &what, &a, &b, &c, &K, &r) == 6) {
        if (what == 's') {                                            // rows before an adapter, to a slice, all rows
            std::printf("%d", more_slices(c, b));
            for (int k = 1; k <= more_slices(c, b); ++k) std::printf(" %d", slice_at_place(k, a, b));
            std::printf("\n");
        } else {                                                      // segments, adapters, rows, long side, rank: the launch's rows and how many
            const GradientForm form = gradient_form_of(APB_BF16, a, b, c, K, r);      // ... of its workgroups may have nothing to do
            const int each = gradient_rows(a, b, c, K, r), tiles = (r + 16 * form.jt - 1) / (16 * form.jt);
            const long long groups = (long long)((K + 16 * form.nc - 1) / (16 * form.nc)) * tiles;
            const int firsts = gradient_by_segment(a, b, K, r) ? a : b;
            const bool by_slice = gradient_by_slice(firsts, c, each, groups);
            const long long more = by_slice ? more_slices(c, each) : (long long)firsts * ((c - 1) / each);
            std::printf("%lld %lld %lld %d\n", (firsts + more) * tiles + 1024, more * groups, more_slices(c, each) * groups, by_slice);
        }
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    at = tmp_path_factory.mktemp("slices")
    src, exe = at / "slices.cpp", at / "slices"
    src.write_text(SLICES)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-ftrapv", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2306_08960_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def answers(questions):
        text = "\n".join(" ".join(map(str, q)) for q in questions)
        p = subprocess.run([str(exe)], input=text, stdout=subprocess.PIPE, text=True, check=True, timeout=60)
        return [list(map(int, line.split())) for line in p.stdout.splitlines()]
    return answers


def test_no_more_idle_workgroups_than_a_few(ask):
    """However many adapters there are: as many workgroups beside their first slices' as there can be slices, or few."""
    g = np.random.default_rng(2)
    sizes = [(int(np.exp(g.uniform(0, 8.3))), int(np.exp(g.uniform(0, 8.3))), int(np.exp(g.uniform(0, 16.6))), int(np.exp(g.uniform(0, 11))),
              int(g.integers(1, 257))) for _ in range(3000)] + [(4096, 4096, 1 << 24, 1 << 22, 256), (1, 1, 1, 1, 1), (256, 256, 65536, 4096, 16)]
    seen = set()
    for (rows, extra, useful, by_slice), size in zip(ask([("w", *s) for s in sizes]), sizes):
        assert rows <= 65535 and extra <= max(useful, 3072), size
        seen.add(by_slice)
    assert seen == {0, 1}


def test_every_slice_has_one_workgroup(ask):
    """First slices have one for each adapter; the others one place each among M / each, and no place stands for two."""
    g = np.random.default_rng(1)
    for case in range(150):
        L, each = int(g.integers(1, 30)), int(g.choice([1, 2, 3, 64, 128, 320]))
        rows = np.where(g.random(L) < 0.3, 0, np.exp(g.uniform(0, 7, L))).astype(int)
        rows[g.integers(L)] = int(g.choice([1, each, each + 1, 3 * each, 3 * each - 1]))
        behind = int(g.integers(0, 300))                             # (rows of no adapter)
        before, M = np.concatenate([[0], np.cumsum(rows)]), int(rows.sum()) + behind
        answers = ask([("s", int(b), each, M, 1, 1) for b in before[:-1]])
        taken, places = [], answers[0][0]
        assert places * each < M
        for k in range(1, places + 1):
            a = int(np.searchsorted(before, k * each, side="right")) - 1
            if a < L and 0 < answers[a][k] < -(-int(rows[a]) // each):
                taken.append((a, answers[a][k]))
        assert sorted(taken) == [(a, z) for a in range(L) for z in range(1, -(-int(rows[a]) // each))]


# ---- sizes beyond 32 bits: refused, not cut to what is left of them ---------------------------------------------------------

def _vast(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta").as_subclass(_On)


BIG = (1 << 32) + 3
VAST = [
    lambda b: b.apb_mx8_quantize(_vast(BIG, 2)), lambda b: b.apb_mx8_quantize(_vast(2, BIG)),
    lambda b: b.apb_mx8_dequantize(_vast(BIG * 33, dtype=torch.uint8), BIG, 32), lambda b: b.alloc_mx8(BIG, 2, device="meta"),
    lambda b: b.apb_gated_forward(_vast(BIG, 2)), lambda b: b.apb_gated_backward(_vast(BIG, 2), _vast(BIG, 1)),
    lambda b: b.apb_gated_backward(_vast(2 * BIG * 33, dtype=torch.uint8), _vast(BIG, 1)),
    lambda b: b.apb_mx4_gated_linear(_vast(BIG, 32), _vast(2 * 136, dtype=torch.uint8), 1),
    lambda b: b.apb_mx4_gated_linear(_vast(4, 32), _vast(2 * 136, dtype=torch.uint8), 1, rows_from=_vast(BIG, dtype=torch.int32)),
    lambda b: b.apb_mx4_gated_linear(_vast(4, 32), _vast(BIG * 2 * 136, dtype=torch.uint8), 1, offsets=_vast(BIG + 1, dtype=torch.int32)),
    lambda b: b.apb_adapter_down(_vast(BIG, 8), _vast(1, 2, 8), adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_down(_vast(4, 8), _vast(BIG, 2, 8), adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_down(_vast(4, 8), _vast(1, BIG, 8), adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_down(_vast(4, 8), _vast(1, 2, 8), _vast(BIG + 1, dtype=torch.int32), _vast(BIG, dtype=torch.int32)),
    lambda b: b.apb_adapter_up(_vast(1, BIG, 2, dtype=torch.float32), _vast(1, 2, 8), adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_up(_vast(1, 4, BIG, dtype=torch.float32), _vast(1, BIG, 8), adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_up(_vast(BIG, 4, 2, dtype=torch.float32), _vast(1, 2, 8), adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_gradient(_vast(1, BIG, 2, dtype=torch.float32), _vast(BIG, 8), 1, adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_gradient(_vast(1, BIG, 2, dtype=torch.float32), _vast(BIG * 33, dtype=torch.uint8), 1, K=8, adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_gradient(_vast(1, 4, BIG, dtype=torch.float32), _vast(4, 8), 1, adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_gradient(_vast(1, 4, 2, dtype=torch.float32), _vast(4, 8), BIG, adapter=_vast(1, dtype=torch.int32)),
    lambda b: b.apb_adapter_gradient(_vast(1, 4, 2, dtype=torch.float32), _vast(4 * 33, dtype=torch.uint8), 1, K=BIG, adapter=_vast(1, dtype=torch.int32)),
]


@needs_lib
@pytest.mark.parametrize("at", range(len(VAST)))
def test_no_size_is_cut_to_32_bits(monkeypatch, at):
    from paper_2306_08960_amd import binding
    real, launched = binding.load(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes") or name.endswith("_parts") or name == "apb_strerror":
                return getattr(real, name)
            return lambda *args: launched.append(name) or 0
    monkeypatch.setattr(binding, "load", Library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    with pytest.raises((binding.ApbError, ValueError)):
        VAST[at](binding)
    assert not launched
    with pytest.raises((binding.ApbError, ValueError)):
        binding.apb_mx4_gated_gemm(_vast(BIG * 136, dtype=torch.uint8), _vast(2 * 136, dtype=torch.uint8), BIG, 1, 32)
    with pytest.raises((binding.ApbError, ValueError)):
        binding.apb_mx4_gated_gemm(_vast(136, dtype=torch.uint8), _vast(BIG * 2 * 136, dtype=torch.uint8), 1, BIG, 32)
    assert not launched


@needs_lib
def test_sizes_are_asked_for_whole():
    from paper_2306_08960_amd import binding as b
    assert b.apb_mx8_bytes(BIG, 32) == 0 and b.apb_mx8_bytes(32, BIG) == 0
    for i in range(4):
        assert b.apb_adapter_parts(*[BIG if k == i else 4 for k in range(4)]) == 0
    for i in range(5):
        assert b.apb_adapter_gradient_workspace_bytes(*[BIG if k == i else v for k, v in enumerate((1, 1, 5000, 64, 4))]) == 0
    for i in range(1, 5):
        assert b.apb_mx4_gated_linear_scratch_bytes(True, *[BIG if k == i else v for k, v in enumerate((0, 2, 500, 4096, 4096)) if k]) == 0
