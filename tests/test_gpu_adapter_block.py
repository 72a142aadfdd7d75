"""Gated blocks, 8-bit checkpoints and adapters together, as examples/adapter_block.py uses them: against the same block in
float64, against differences, in captured graphs, on other streams.

Tolerances, fixed before the first run.  In float32 the block's outputs differ from float64's by float32 sums, and where a value
lies so near to a border that it goes to the neighbouring 4- or 8-bit value: relative to the norm of the result a 4-bit step of
1/4 for a share of 1e-5 of the values is 1e-3, so outputs and gradients are held to 4e-3 of their norm.  In bfloat16 each of up to
eight roundings in a row adds 2^-8: 2^-5."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import block_oracle as o
from oracle import mx4_oracle as o4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu

NORM = {torch.float32: 4e-3, torch.bfloat16: 2.0 ** -5, torch.float16: 2.0 ** -5}


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import adapter_block
    return adapter_block


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _q4(x):
    codes, scales = o4.quantize(x.astype(np.float32))
    return o4.values(codes, scales, x.shape[1])


def _q8(x):
    return o.values8(*o.quantize8(x.astype(np.float32)), x.shape[1])


def _block(ex, dtype, K, H, L, r, activation="silu"):
    block = ex.AdapterBlock(K, H, L, r, activation, dtype, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    for name in ("b_gu", "b_d"):
        block.latent[name] = torch.randn(block.latent[name].shape, generator=g, device="cuda") * 0.3
    block.cast()
    return block


def _reference(block, x, dy, which):
    """Everything in float64, from the bytes of the 4-bit weights."""
    apb = sys.modules["adapter_block"].apb
    K, H, L = block.K, block.H, block.L
    f = {k: _np(v) for k, v in block.f.items()}
    s = _np(block.scale)
    wgu, wd = _np(apb.apb_mx4_dequantize(block.q_gu, 2 * H, K)), _np(apb.apb_mx4_dequantize(block.q_d, K, H))
    t_gu = o.down(x, f["a_gu"], which, s)[0]
    gu = _q4(x) @ wgu.T + o.up(t_gu, f["b_gu"], which)
    h = o.act(gu[:, :H], block.activation)[0] * gu[:, H:]
    t_d = o.down(h, f["a_d"], which, s)[0]
    y = _q4(h) @ wd.T + o.up(t_d, f["b_d"], which)
    dt_d = o.down(dy, f["b_d"], which, s)[0]
    dh = dy @ wd + o.up(dt_d, f["a_d"], which)
    g8, u8 = _q8(gu[:, :H]), _q8(gu[:, H:])
    v, d, _, _ = o.act(g8, block.activation)
    dgu = np.concatenate([dh * u8 * d, dh * v], 1)
    dt_gu = o.down(dgu, f["b_gu"], which, s)[0]
    return y, dgu @ wgu + o.up(dt_gu, f["a_gu"], which), {
        "b_d": o.gradient(t_d, dy, which, L), "a_d": o.gradient(dt_d, v * u8, which, L),
        "b_gu": o.gradient(t_gu, dgu, which, L), "a_gu": o.gradient(dt_gu, _q8(x), which, L)}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K,H,L,r,activation", [(96, 160, 3, 4, "silu"), (130, 75, 2, 17, "gelu"), (256, 512, 4, 33, "relu")])
def test_block_against_float64(ex, K, H, L, r, activation, dtype):
    block = _block(ex, dtype, K, H, L, r, activation)
    lengths, adapters = [50, 0, 1, 90, 33, 17], [0, 1, -1, L - 1, 1, 0]
    M = sum(lengths) + 9                                             # (nine rows behind the last sequence)
    seg = ex.segments(lengths, adapters)
    g = torch.Generator(device="cuda").manual_seed(K)
    x, dy = torch.randn(M, K, generator=g, device="cuda").to(dtype), (torch.randn(M, K, generator=g, device="cuda") * 0.1).to(dtype)
    which = o.rows_by_adapter(seg["offsets"].tolist(), adapters, M, L)
    want_y, want_dx, want = _reference(block, _np(x), _np(dy), which)
    y, kept = block.forward(x, seg)
    dx, grad = block.backward(dy, kept)
    near = lambda a, b: np.linalg.norm(_np(a) - b) <= NORM[dtype] * np.linalg.norm(b)
    assert near(y, want_y) and near(dx, want_dx)
    for name in want:
        assert grad[name].dtype == torch.float32 and near(grad[name], want[name]), name
    assert torch.equal(block.serve(x, seg), y)


def test_block_against_differences(ex):
    """<Y, dY> is linear in the second side of the last adapter: its gradient is the difference over any step.  Whole numbers all
    the way after the activation, so only the sums over 100 rows and 96 columns are rounded."""
    block = _block(ex, torch.float32, 96, 160, 3, 4)
    seg = ex.segments([40, 60], [2, 0])
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = torch.randn(100, 96, generator=g, device="cuda"), torch.randn(100, 96, generator=g, device="cuda")
    way = torch.randn(block.latent["b_d"].shape, generator=g, device="cuda")
    y, kept = block.forward(x, seg)
    grad = block.backward(dy, kept)[1]["b_d"]
    loss = []
    for sign in (1.0, -1.0):
        block.latent["b_d"] += sign * way
        block.cast()
        loss.append((block.forward(x, seg)[0].double() * dy.double()).sum().item())
        block.latent["b_d"] -= sign * way
    slope, want = (loss[0] - loss[1]) / 2, (grad.double() * way.double()).sum().item()
    # every y is off by at most 300 * 2^-23 of the magnitudes it is a sum of, below 50 each
    assert abs(slope - want) <= 300 * 2.0 ** -23 * 50 * dy.abs().sum().item()
    assert bool((grad[1] == 0).all())


def test_serving_a_token_of_every_request(ex):
    block = _block(ex, torch.bfloat16, 256, 512, 4, 16)
    g = torch.Generator(device="cuda").manual_seed(2)
    adapters = [0, -1, 3, 1, 1, 2, 0, 3, -1, 2, 1]
    x = torch.randn(len(adapters), 256, generator=g, device="cuda").bfloat16()
    together = block.serve(x, ex.segments([1] * len(adapters), adapters))
    bare = block.serve(x)
    for i, a in enumerate(adapters):
        alone = block.serve(x[i:i + 1], ex.segments([1], [a]))
        # (other kernels may sum in another order: bfloat16's roundings, and 4-bit values beside a border)
        assert (alone[0].float() - together[i].float()).norm() <= NORM[torch.bfloat16] * together[i].float().norm()
        if a < 0:
            assert (bare[i].float() - together[i].float()).norm() <= NORM[torch.bfloat16] * together[i].float().norm()


def test_captured_steps(ex):
    """A step of tuning and one of serving in graphs, replayed with other inputs and eager work between the replays."""
    block = _block(ex, torch.bfloat16, 256, 512, 4, 16)
    seg, one = ex.segments([300, 0, 200, 100], [0, 1, 3, -1]), ex.segments([1] * 5, [3, 0, -1, 2, 2])
    g = torch.Generator(device="cuda").manual_seed(7)
    x, dy = torch.zeros(600, 256, device="cuda").bfloat16(), torch.zeros(600, 256, device="cuda").bfloat16()
    tokens = torch.zeros(5, 256, device="cuda").bfloat16()

    def tune():
        y, kept = block.forward(x, seg)
        dx, grad = block.backward(dy, kept)
        return [y, dx, *grad.values()]

    tune(), block.serve(tokens, one), block.serve(tokens)            # (what a first call sets up)
    torch.cuda.synchronize()
    graphs = []
    for call in (tune, lambda: [block.serve(tokens, one)], lambda: [block.serve(tokens)]):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out, call))
    for _ in range(4):
        for t in (x, dy, tokens):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        for graph, out, call in graphs:
            graph.replay()
            got = [t.clone() for t in out]
            torch.cuda.synchronize()
            for a, b in zip(got, call()):
                assert torch.equal(a, b)


def test_another_stream(ex):
    apb = ex.apb
    block = _block(ex, torch.bfloat16, 256, 512, 4, 16)
    seg = ex.segments([100, 28], [2, 0])
    x = torch.randn(128, 256, device="cuda").bfloat16()
    f = block.f
    gu = apb.apb_mx4_linear(x, block.q_gu, 1024)
    t = apb.apb_adapter_down(x, f["a_gu"], scale=block.scale, **seg)
    up = apb.apb_adapter_up(t, f["b_gu"], Y0=gu, **seg)
    saved = apb.alloc_mx8(256, 512)
    h = apb.apb_gated_forward(up, saved=saved)
    d = apb.apb_gated_backward(saved, h)
    da = apb.apb_adapter_gradient(t, x, 4, **seg)
    direct = apb.apb_mx4_gated_linear(x, block.q_gu, 512)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for use in (dict(stream=side), dict()):
        with torch.cuda.stream(torch.cuda.current_stream() if use else side):
            t2 = apb.apb_adapter_down(x, f["a_gu"], scale=block.scale, **seg, **use)
            up2 = apb.apb_adapter_up(t2, f["b_gu"], Y0=gu, **seg, **use)
            s2 = torch.empty_like(saved)
            side.wait_stream(torch.cuda.default_stream())
            h2 = apb.apb_gated_forward(up2, saved=s2, **use)
            d2 = apb.apb_gated_backward(s2, h2, **use)
            da2 = apb.apb_adapter_gradient(t2, x, 4, **seg, **use)
            x8 = apb.apb_mx8_quantize(x, **use)
            x2 = apb.apb_mx8_dequantize(x8, 128, 256, torch.bfloat16, **use)
            direct2 = apb.apb_mx4_gated_linear(x, block.q_gu, 512, **use)
        side.synchronize()
        for a, b in ((t, t2), (up, up2), (saved, s2), (h, h2), (d, d2), (da, da2), (direct, direct2)):
            assert torch.equal(a, b)
        assert torch.equal(x2, apb.apb_mx8_dequantize(apb.apb_mx8_quantize(x), 128, 256, torch.bfloat16))


def test_example_runs(ex):
    losses, batch, step = ex.main(steps=3)
    assert len(losses) == 3 and all(np.isfinite(losses))
    assert (batch.float() - step.float()).norm() <= NORM[torch.bfloat16] * batch.float().norm()


def test_another_device_is_refused(monkeypatch):
    """Kernels go to the current device: with another one current (as far as the binding is told) no call gets as far as a launch."""
    from paper_2306_08960_amd import binding as b
    x, A = torch.randn(4, 64, device="cuda"), torch.randn(1, 3, 64, device="cuda")
    w, seg = b.apb_mx4_quantize(torch.randn(64, 64, device="cuda")), dict(adapter=torch.zeros(1, dtype=torch.int32, device="cuda"))
    T, x8, saved, x4 = b.apb_adapter_down(x, A, **seg), b.apb_mx8_quantize(x), b.alloc_mx8(8, 32), b.apb_mx4_quantize(x)
    calls = [lambda: b.apb_mx8_quantize(x), lambda: b.apb_mx8_dequantize(x8, 4, 64), lambda: b.apb_mx4_gated_gemm(x4, w, 4, 32, 64),
             lambda: b.apb_mx4_gated_linear(x, w, 32), lambda: b.apb_gated_forward(x, saved=saved),
             lambda: b.apb_gated_backward(saved, x[:, :32]), lambda: b.apb_adapter_down(x, A, **seg), lambda: b.apb_adapter_up(T, A, **seg),
             lambda: b.apb_adapter_gradient(T, x, 1, **seg)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    here = torch.cuda.current_device()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: here + 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
