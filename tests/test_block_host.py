"""Gated blocks, 8-bit checkpoints and adapters without a GPU: pins of the oracle, sizes, and the refusals of every entry point."""
import ctypes
import os

import numpy as np
import pytest

from oracle import block_oracle as o

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2306_08960_amd", "libapb.so")


# ---- the oracle ------------------------------------------------------------------------------------------------------

def test_eight_bits_by_hand():
    x = np.zeros((1, 40), np.float32)
    x[0, :5] = 1.0, 0.5, 1.0 / 64, 1.5 / 64, 2.5 / 64                # e = -6: steps of 1/64, ties to even
    x[0, 32:35] = 255.0, 254.0, -254.9                               # e = 1: 127.5 -> 128 -> 127
    codes, scales = o.quantize8(x)
    assert scales.tolist() == [[127 - 6, 127 + 1]]
    assert codes[0, :5].tolist() == [64, 32, 1, 2, 2] and codes[0, 32:35].tolist() == [127, 127, -127]
    assert np.array_equal(o.values8(codes, scales, 40)[0, 32:35], [254.0, 254.0, -254.0])
    assert np.all(codes[0, 40:] == 0)


def test_eight_bits_error():
    x = (np.random.default_rng(0).standard_normal((50, 100)) * np.exp2(np.random.default_rng(1).integers(-20, 20, (50, 1)))).astype(np.float32)
    codes, scales = o.quantize8(x)
    back = o.values8(codes, scales, 100)
    pad = np.zeros((50, 128))
    pad[:, :100] = x
    top = np.repeat(np.abs(pad.reshape(50, 4, 32)).max(2), 32, 1)[:, :100]
    assert np.all(np.abs(back - x) <= top * 2.0 ** -7 + 1e-300)


def test_eight_bits_specials():
    x = np.zeros((4, 32), np.float32)
    x[0, 3], x[1, 3] = np.inf, np.nan
    x[2, 0], x[3, 0] = 3.4028235e38, 1e-45
    codes, scales = o.quantize8(x)
    assert scales[:, 0].tolist() == [255, 255, 248, 0]
    assert np.isnan(o.values8(codes, scales, 32)[:2]).all()
    assert codes[2, 0] == 127 and codes[3, 0] == 0
    assert np.array_equal(o.unpack8(o.pack8(codes, scales), 4, 32)[1], scales)


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
def test_activations(kind):
    x = np.concatenate([np.linspace(-30, 30, 1201), [1e4, -1e4, 1e30, -1e30]])
    x = x[x != 0]
    v, d, _, _ = o.act(x, kind)
    assert np.isfinite(v).all() and np.isfinite(d).all()
    if kind == "gelu":
        tanh = 0.5 * x * (1 + np.tanh(o.ROOT * (x + 0.044715 * x ** 3)))
        assert np.allclose(v, tanh, rtol=1e-6, atol=1e-12)
    near = np.abs(x) < 31
    h = 1e-5
    diff = (o.act(x[near] + h, kind)[0] - o.act(x[near] - h, kind)[0]) / (2 * h)
    assert np.allclose(d[near], diff, rtol=1e-6, atol=1e-8)
    assert o.act(np.array([np.inf]), kind)[0][0] == np.inf and o.act(np.array([-np.inf]), kind)[0][0] == 0
    assert o.act(np.array([np.inf]), kind)[1][0] == 1 and o.act(np.array([-np.inf]), kind)[1][0] == 0


def test_adapter_gradients_of_the_oracle_by_differences():
    g = np.random.default_rng(3)
    M, K, N, r, L = 9, 7, 5, 3, 2
    x, A, B, dy = g.standard_normal((M, K)), g.standard_normal((L, r, K)), g.standard_normal((L, r, N)), g.standard_normal((M, N))
    scale, offsets, adapter = np.array([0.5, 2.0]), [0, 2, 2, 6, 8], [1, 0, -1, 0]
    which = o.rows_by_adapter(offsets, adapter, M, L)
    loss = lambda x, A, B: float((o.up(o.down(x, A, which, scale)[0], B, which) * dy).sum())
    T, dT = o.down(x, A, which, scale)[0], o.down(dy, B, which, scale)[0]
    for name, want in (("x", o.up(dT, A, which)), ("A", o.gradient(dT, x, which, L)), ("B", o.gradient(T, dy, which, L))):
        p = dict(x=x, A=A, B=B)
        for at in np.ndindex(p[name].shape):
            e = np.zeros_like(p[name])
            e[at] = 1e-4
            diff = (loss(**{**p, name: p[name] + e}) - loss(**{**p, name: p[name] - e})) / 2e-4
            assert abs(diff - want[at]) < 1e-7


# ---- sizes and refusals ----------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def b():
    if not os.path.exists(LIB):
        pytest.skip("libapb.so not built")
    from paper_2306_08960_amd import binding
    binding.load()
    return binding


P, Q, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 21), ctypes.c_void_p((1 << 20) + 2)     # never followed: every call fails before


def test_mx8_bytes(b):
    assert b.apb_mx8_bytes(1, 1) == 33 and b.apb_mx8_bytes(3, 32) == 99 and b.apb_mx8_bytes(3, 33) == 198
    assert b.apb_mx8_bytes(0, 5) == 0 and b.apb_mx8_bytes(5, 0) == 0 and b.apb_mx8_bytes(1, (1 << 22) + 1) == 0
    assert b.apb_mx8_bytes((1 << 30) - 64, 32) == ((1 << 30) - 64) * 33 and b.apb_mx8_bytes((1 << 30) - 63, 32) == 0
    for rows, K in ((0, 4), (4, 0), (1, (1 << 22) + 1), ((1 << 30) - 63, 32)):
        with pytest.raises(b.ApbError):
            b.alloc_mx8(rows, K)
    for rows, K in ((1, 1), (3, 32), (7, 517), (2, 1 << 22)):
        assert b.alloc_mx8(rows, K, device="meta").numel() == b.apb_mx8_bytes(rows, K)


def test_mx8_refusals(b):
    lib = b.load()
    for f, args in ((lib.apb_mx8_quantize, lambda X=P, t=1, ld=40, rows=4, K=40, m=P: (X, t, ld, rows, K, m, None)),
                    (lib.apb_mx8_dequantize, lambda X=P, t=1, ld=40, rows=4, K=40, m=P: (m, rows, K, t, X, ld, None))):
        assert f(*args(X=None)) == b.APB_ERR_NULL and f(*args(m=None)) == b.APB_ERR_NULL
        assert f(*args(t=3)) == b.APB_ERR_TYPE and f(*args(t=-1)) == b.APB_ERR_TYPE
        assert f(*args(ld=39)) == b.APB_ERR_SHAPE and f(*args(rows=0)) == b.APB_ERR_SHAPE and f(*args(K=0)) == b.APB_ERR_SHAPE
        assert f(*args(m=ODD)) == b.APB_ERR_ALIGN and f(*args(X=ODD, t=0)) == b.APB_ERR_ALIGN


def test_gated_product_refusals(b):
    lib = b.load()

    def gemm(A=P, W=P, off=None, E=1, M=8, N=40, K=64, act=0, t=1, Y=P, ld=40, saved=None):
        return lib.apb_mx4_gated_gemm(A, W, off, E, M, N, K, act, t, Y, ld, saved, None)

    def linear(X=P, xt=1, ldx=64, rows_in=8, rows=None, W=P, off=None, E=1, M=8, N=40, K=64, act=0, scratch=P, t=1, Y=P, ld=40, saved=None):
        return lib.apb_mx4_gated_linear(X, xt, ldx, rows_in, rows, W, off, E, M, N, K, act, scratch, t, Y, ld, saved, None)

    for f in (gemm, linear):
        for k in ("W", "Y"):
            assert f(**{k: None}) == b.APB_ERR_NULL
            assert f(**{k: ODD}, t=0) == b.APB_ERR_ALIGN
        assert f(t=3) == b.APB_ERR_TYPE and f(act=3) == b.APB_ERR_VALUE and f(act=-1) == b.APB_ERR_VALUE
        for k in ("M", "N", "K", "E"):
            assert f(**{k: 0}) == b.APB_ERR_SHAPE
        assert f(ld=39) == b.APB_ERR_SHAPE and f(E=2) == b.APB_ERR_SHAPE and f(off=P, E=1025) == b.APB_ERR_SHAPE
        assert f(N=1 << 30, ld=1 << 30) == b.APB_ERR_SHAPE and f(M=(1 << 30) + 1, N=1) == b.APB_ERR_SHAPE
        assert f(saved=ODD) == b.APB_ERR_ALIGN and f(off=ODD) == b.APB_ERR_ALIGN
    assert gemm(A=None) == b.APB_ERR_NULL and gemm(A=ODD) == b.APB_ERR_ALIGN
    assert linear(X=None) == b.APB_ERR_NULL and linear(scratch=None) == b.APB_ERR_NULL and linear(xt=3) == b.APB_ERR_TYPE
    assert linear(ldx=63) == b.APB_ERR_SHAPE and linear(rows_in=7) == b.APB_ERR_SHAPE and linear(rows_in=0, rows=P) == b.APB_ERR_SHAPE
    assert linear(X=ODD, xt=0) == b.APB_ERR_ALIGN and linear(scratch=ODD) == b.APB_ERR_ALIGN


def test_gated_scratch(b):
    s = b.apb_mx4_gated_linear_scratch_bytes
    assert s(False, 1, 1, 4096, 4096) == 0 and s(False, 1, 1, 4096, 4096, True) == b.apb_mx4_bytes(1, 4096)
    assert s(False, 1, 500, 4096, 4096) == b.apb_mx4_bytes(500, 4096) and s(False, 1, 0, 4096, 4096) == 0
    assert s(False, 1, 500, 1 << 30, 4096) == 0


def test_gated_activation_refusals(b):
    lib = b.load()

    def forward(GU=P, t=1, ldgu=80, M=8, N=40, act=0, Y=P, ld=40, saved=None):
        return lib.apb_gated_forward(GU, t, ldgu, M, N, act, Y, ld, saved, None)

    def backward(GU=P, gt=1, ldgu=80, dY=P, t=1, lddy=40, M=8, N=40, act=0, dGU=Q, lddgu=80, Y=None, ld=40):
        return lib.apb_gated_backward(GU, gt, ldgu, dY, t, lddy, M, N, act, dGU, lddgu, Y, ld, None)

    for f in (forward, backward):
        assert f(GU=None) == b.APB_ERR_NULL and f(t=3) == b.APB_ERR_TYPE and f(act=3) == b.APB_ERR_VALUE
        assert f(M=0) == b.APB_ERR_SHAPE and f(N=0) == b.APB_ERR_SHAPE and f(ldgu=79) == b.APB_ERR_SHAPE and f(M=-1) == b.APB_ERR_SHAPE
        assert f(Y=P, ld=39) == b.APB_ERR_SHAPE and f(Y=ODD, t=0) == b.APB_ERR_ALIGN
        assert f(N=(1 << 22) + 1, ldgu=1 << 24, ld=1 << 24) == b.APB_ERR_SHAPE
    assert forward(Y=None) == b.APB_ERR_NULL and forward(saved=ODD) == b.APB_ERR_ALIGN and forward(GU=ODD, t=0) == b.APB_ERR_ALIGN
    assert backward(dY=None) == b.APB_ERR_NULL and backward(dGU=None) == b.APB_ERR_NULL and backward(gt=4) == b.APB_ERR_TYPE
    assert backward(lddy=39) == b.APB_ERR_SHAPE and backward(lddgu=79) == b.APB_ERR_SHAPE
    assert backward(GU=ODD, gt=3) == b.APB_ERR_ALIGN and backward(GU=ODD, gt=0) == b.APB_ERR_ALIGN
    assert backward(dGU=P, gt=3) == b.APB_ERR_SHAPE and backward(dGU=P, gt=2) == b.APB_ERR_SHAPE      # (GU itself)
    assert backward(dGU=P, lddgu=96) == b.APB_ERR_SHAPE
    assert backward(dY=ODD, t=0) == b.APB_ERR_ALIGN and backward(dGU=ODD, t=0) == b.APB_ERR_ALIGN


def test_adapter_refusals(b):
    lib = b.load()

    def down(X=P, t=1, ldx=64, A=P, off=P, ad=P, scale=None, S=3, L=2, M=20, K=64, r=8, T=P):
        return lib.apb_adapter_down(X, t, ldx, A, off, ad, scale, S, L, M, K, r, T, None)

    def up(T=P, parts=1, A=P, t=1, off=P, ad=P, S=3, L=2, M=20, K=64, r=8, Y0=None, ld0=64, X=P, ldx=64):
        return lib.apb_adapter_up(T, parts, A, t, off, ad, S, L, M, K, r, Y0, ld0, X, ldx, None)

    def gradient(T=P, parts=1, X=P, t=1, ldx=64, off=P, ad=P, S=3, L=2, M=20, K=64, r=8, A=P, ws=None, wb=0):
        return lib.apb_adapter_gradient(T, parts, X, t, ldx, off, ad, S, L, M, K, r, A, ws, wb, None)

    odd1 = ctypes.c_void_p((1 << 20) + 1)
    for f in (down, up, gradient):
        for k in ("X", "A", "T"):
            assert f(**{k: None}) == b.APB_ERR_NULL
            assert f(**{k: ODD}, t=0) == b.APB_ERR_ALIGN or k == "A" and f is gradient
        for k, bad in (("S", (0, 4097)), ("L", (0, 4097)), ("M", (0, (1 << 24) + 1)), ("K", (0, (1 << 22) + 1)), ("r", (0, 257))):
            for v in bad:
                assert f(**{k: v}) == b.APB_ERR_SHAPE
        assert f(ldx=63) == b.APB_ERR_SHAPE and f(t=4) == b.APB_ERR_TYPE
        assert f(off=None) == b.APB_ERR_SHAPE and f(ad=None) == b.APB_ERR_SHAPE
        assert f(off=odd1) == b.APB_ERR_ALIGN and f(ad=odd1) == b.APB_ERR_ALIGN
    assert down(t=3) == b.APB_ERR_TYPE and up(t=3) == b.APB_ERR_TYPE and down(scale=ODD) == b.APB_ERR_ALIGN
    for f in (up, gradient):
        assert f(parts=0) == b.APB_ERR_SHAPE and f(parts=9) == b.APB_ERR_SHAPE
    assert up(Y0=P, ld0=63) == b.APB_ERR_SHAPE and up(Y0=P, ld0=65, X=P) == b.APB_ERR_SHAPE
    assert gradient(t=3, X=ODD) == b.APB_ERR_ALIGN and gradient(A=ODD) == b.APB_ERR_ALIGN and gradient(ws=ODD) == b.APB_ERR_ALIGN
    assert b.apb_adapter_parts(0, 4, 4, 4) == 0 and b.apb_adapter_parts(1, 1, 1, 1) == 1 and b.apb_adapter_parts(1, 1, 1, 257) == 0
    assert b.apb_adapter_gradient_workspace_bytes(1, 0, 4, 4, 4) == 0 and b.apb_adapter_gradient_workspace_bytes(1, 1, 1, 1, 1) == 0
