"""Gated blocks, 8-bit checkpoints and adapters: what NaN, infinities and memory beside the operands may reach, and the precision that
the header promises for single terms."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2306_08960_amd import binding
    binding.load()
    return binding


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_nan_gate_reaches_its_gradients(b, t, kind):
    """A gate that is NaN has NaN gradients, and nobody else has: from the float matrix one value, from 8 bits its block."""
    M, N = 5, 70
    g = torch.Generator(device="cuda").manual_seed(3)
    gu = torch.randn(M, 2 * N, generator=g, device="cuda").to(TYPE[t])
    dy = torch.ones(M, N, device="cuda").to(TYPE[t])
    gu[1, 5], gu[3, 66] = float("nan"), float("nan")
    saved = b.alloc_mx8(2 * M, N)
    b.apb_gated_forward(gu, kind, saved=saved)
    one = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    one[1, 5] = one[3, 66] = True
    block = torch.zeros_like(one)
    block[1, :32] = block[3, 64:] = True
    for source, want in ((gu, one), (saved, block)):
        y = torch.empty(M, N, dtype=TYPE[t], device="cuda")
        d = b.apb_gated_backward(source, dy, kind, Y=y)
        for got in (y, d[:, :N], d[:, N:]):
            assert torch.equal(torch.isnan(got), want)
    gu[1, 5] = gu[3, 66] = 0.0
    gu[2, N + 7] = float("nan")                                      # an up projection that is NaN: Y and dG
    one[:] = False
    one[2, 7] = True
    d = b.apb_gated_backward(gu, dy, kind, Y=y)
    assert torch.equal(torch.isnan(y), one) and torch.equal(torch.isnan(d[:, :N]), one) and bool(torch.isfinite(d[:, N:]).all())


def test_product_beyond_the_8_bit_form(b):
    """More rows than both projections could be saved of in 8 bits, and more than 2^34 outputs: the last rows against themselves alone."""
    M, N, K, tail = 1 << 20, 16385, 32, 300
    assert b.apb_mx8_bytes(2 * M, N) == 0
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    w4 = b.apb_mx4_quantize(torch.randn(2 * N, K, generator=g, device="cuda"))
    last = b.apb_mx4_gated_linear(x[M - tail:], w4, N)
    y = b.apb_mx4_gated_linear(x, w4, N)
    assert torch.equal(y[M - tail:], last)
    assert bool(torch.isfinite(last).all()) and int((last != 0).sum()) > last.numel() // 2
    y.zero_()
    b.apb_mx4_gated_gemm(b.apb_mx4_quantize(x), w4, M, N, K, Y=y)
    assert torch.equal(y[M - tail:], last)
    with pytest.raises(ValueError):
        b.apb_mx4_gated_linear(x, w4, N, saved=torch.empty(64, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("M,N,E", [(40, 30001, 0), (200, 24600, 0), (512, 8200, 16), (2000, 2111, 64)])
def test_few_rows_and_many_columns(b, M, N, E):
    """The kernel for few rows where tiles would be mostly empty, against the tiles (which a call takes that saves both projections): with
    one block a row every sum is exact, so the two agree to the bit."""
    K = 32
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    w4 = b.apb_mx4_quantize(torch.randn(max(E, 1) * 2 * N, K, generator=g, device="cuda"))
    off = None
    if E:
        off = torch.sort(torch.randint(0, M - 8, (E + 1,), generator=g, device="cuda")).values.int()
        off[0] = 0
    assert b.apb_mx4_gated_linear_scratch_bytes(E > 0, max(E, 1), M, N, K) == 0
    few = b.apb_mx4_gated_linear(x, w4, N, offsets=off)
    tiles = b.apb_mx4_gated_linear(x, w4, N, offsets=off, saved=b.alloc_mx8(2 * M, N))
    assert torch.equal(few, tiles) and bool(torch.isfinite(few).all())
