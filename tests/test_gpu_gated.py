"""8-bit checkpoints and gated blocks through the C ABI against the oracle in float64.

Tolerances, fixed before the first run.
Sums of products of 4-bit values: (K / 16 + 64) * 2^-23 of the sum of the magnitudes, as for the plain products.
The sigmoid s(z): z has up to four rounded factors and constants (5 * 2^-24 relative, which the exponential turns into |z| times
that), the exponential and the reciprocal are off by 2^-23 each, two more roundings: together below 2^-21 (1 + |z|) relative, and
values below 2^-118 may be lost.  act'(x) = s + x s (1 - s) z' is off by that relative to s (1 + |x| z').  Each further product adds
2^-24.  8-bit values: half a step, a whole one beyond 126.5 steps.  Outputs are rounded once to their type."""
import numpy as np
import pytest
import torch

import gated_cases as gated
import mx4_tile_cases as cases
from oracle import block_oracle as o
from oracle import mx4_oracle as o4

pytestmark = pytest.mark.gpu

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {t: torch.finfo(d).eps / 2 for t, d in TYPE.items()}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
ACTS = ["silu", "gelu", "relu"]


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2306_08960_amd import binding
    binding.load()
    return binding


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _in(a, t):
    x = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPE[t])
    return x.cuda(), x.float().numpy()


def _check(got, want, tol, t):
    tol = tol + HALF_ULP[t] * 1.001 * (np.abs(want) + tol) + TINY[t]
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (at, got[at], want[at], tol[at])


def _acts(seed, M, K):
    g = np.random.default_rng(seed)
    return (g.standard_normal((M, K)) * np.exp(g.standard_normal(K))).astype(np.float32)


def _wide(x, extra=5, at=3, fill=99.0):
    """The same matrix as a window of a wider one."""
    w = torch.full((x.shape[0], x.shape[1] + extra), fill, dtype=x.dtype, device="cuda")
    w[:, at:at + x.shape[1]] = x
    return w[:, at:at + x.shape[1]]


# ------------------------------------------------------------------------------------------ 8-bit checkpoints

@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 31), (3, 32), (5, 33), (2, 255), (33, 517), (9, 4096), (700, 100)])
def test_mx8_and_back(b, M, K, t):
    x, v = _in(_acts(M + K, M, K), t)
    v = v.copy()
    if M > 1:                                                        # ties and values that go beyond 127 steps
        v[0] = (np.arange(K) % 255 - 127) / 2 * 0.25
        v[0, 0] = 31.9375
        v[1] = 0
        x, v = _in(v, t)
    want = o.quantize8(v)
    for view in (x, _wide(x)):
        mx8 = b.apb_mx8_quantize(view)
        assert np.array_equal(mx8.cpu().numpy(), o.pack8(*want))
    val = o.values8(*want, K)
    for back in TYPE:
        got = b.apb_mx8_dequantize(mx8, M, K, TYPE[back])
        assert torch.equal(got.cpu(), torch.from_numpy(val).to(TYPE[back]))
    frame = torch.full((M, K + 4), 7.0, dtype=TYPE[t], device="cuda")
    b.apb_mx8_dequantize(mx8, M, K, X=frame[:, 2:K + 2])
    assert torch.equal(frame[:, 2:K + 2].cpu(), torch.from_numpy(val).to(TYPE[t])) and bool((frame[:, :2] == 7).all() and (frame[:, K + 2:] == 7).all())


def test_mx8_extremes(b):
    x = np.zeros((7, 64), np.float32)
    x[0, :40], x[0, 1] = 3.4028235e38, -3.4028235e38
    x[1, :4] = 1e-45, -3e-39, 1.1754944e-38, 5e-39
    x[2, 3], x[2, 40] = np.inf, 1.0
    x[3, 3], x[3, 40] = np.nan, -1.0
    x[4, 0], x[4, 1] = -np.inf, 5.0
    x[5, :2] = 1e30, 1e-30
    x[6, :] = -0.0
    want = o.quantize8(x)
    mx8 = b.apb_mx8_quantize(torch.from_numpy(x).cuda())
    assert np.array_equal(mx8.cpu().numpy(), o.pack8(*want))
    assert np.array_equal(b.apb_mx8_dequantize(mx8, 7, 64).cpu().numpy(), o.values8(*want, 64).astype(np.float32), equal_nan=True)


# ------------------------------------------------------------------------------------------ the activation by itself

def _act_error(x, kind):
    v, d, z, dz = o.act(x, kind)
    s = np.where(x != 0, np.abs(v / np.where(x != 0, x, 1)), 0.5)
    rel = 2.0 ** -21 * (1 + z)
    if kind == "relu":
        return v, d, np.zeros_like(v), np.zeros_like(v)
    return v, d, rel * np.abs(v) + 2.0 ** -118, rel * s * (1 + np.abs(x) * dz) + 2.0 ** -118


def _expect(g, u, dy, kind):
    """{name: (value, tolerance)} of y, dg, du from values that are exact."""
    v, d, ev, ed = _act_error(g, kind)
    k = 2.0 ** -23
    return {"y": (v * u, np.abs(u) * ev + k * np.abs(v * u)),
            "dg": (dy * u * d, np.abs(dy * u) * ed + 2 * k * np.abs(dy * u * d)),
            "du": (dy * v, np.abs(dy) * ev + k * np.abs(dy * v))}


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N", [(1, 1), (3, 31), (2, 32), (65, 33), (7, 517), (130, 1000)])
def test_activation_and_gradients(b, M, N, t, kind):
    gu, v = _in(_acts(M * 7 + N, M, 2 * N) * 2, t)
    dy, dv = _in(_acts(M + N + 1, M, N), t)
    v, dv = v.astype(np.float64), dv.astype(np.float64)
    saved = b.alloc_mx8(2 * M, N)
    y = b.apb_gated_forward(_wide(gu), kind, saved=saved)
    want = _expect(v[:, :N], v[:, N:], dv, kind)
    _check(_np(y), *want["y"], t)
    both = np.concatenate([v[:, :N], v[:, N:]]).astype(np.float32)
    kept = o.quantize8(both)
    assert np.array_equal(saved.cpu().numpy(), o.pack8(*kept))
    assert torch.equal(y, b.apb_gated_forward(gu, kind))
    q = o.values8(*kept, N)
    for source, (g, u) in ((saved, (q[:M], q[M:])), (_wide(gu), (v[:, :N], v[:, N:]))):
        want = _expect(g, u, dv, kind)
        again = torch.full((M, N + 3), 5.0, dtype=TYPE[t], device="cuda")
        dgu = torch.full((M, 2 * N + 3), 5.0, dtype=TYPE[t], device="cuda")
        b.apb_gated_backward(source, _wide(dy), kind, dGU=dgu[:, 1:2 * N + 1], Y=again[:, 2:N + 2])
        assert bool((dgu[:, 0] == 5).all() and (dgu[:, 2 * N + 1:] == 5).all() and (again[:, :2] == 5).all() and (again[:, N + 2:] == 5).all())
        _check(_np(again[:, 2:N + 2]), *want["y"], t)
        _check(_np(dgu[:, 1:N + 1]), *want["dg"], t)
        _check(_np(dgu[:, N + 1:2 * N + 1]), *want["du"], t)
        assert torch.equal(b.apb_gated_backward(source, dy, kind), dgu[:, 1:2 * N + 1])
    inplace = gu.clone()
    b.apb_gated_backward(inplace, dy, kind, dGU=inplace)
    assert torch.equal(inplace, dgu[:, 1:2 * N + 1])


@pytest.mark.parametrize("kind", ACTS)
def test_activation_over_its_range(b, kind):
    """Gates from the smallest to the largest, infinities and NaN; the gradient also against differences."""
    x = np.concatenate([np.linspace(-100, 100, 2001), 10.0 ** np.arange(-38, 39, 2), -10.0 ** np.arange(-38, 39, 2), [0.0, -0.0]]).astype(np.float32)
    n = len(x)
    gu = torch.from_numpy(np.stack([x, np.ones(n, np.float32)], 1)).cuda()
    one = torch.ones(n, 1, device="cuda")
    y = torch.empty(n, 1, device="cuda")
    dgu = _np(b.apb_gated_backward(gu, one, kind, Y=y))
    want = _expect(x[:, None].astype(np.float64), np.ones((n, 1)), np.ones((n, 1)), kind)
    _check(_np(y), *want["y"], "f32")
    _check(_np(b.apb_gated_forward(gu, kind)), *want["y"], "f32")
    _check(dgu[:, :1], *want["dg"], "f32")
    _check(dgu[:, 1:], *want["du"], "f32")
    # (steps of 0.1 inside -20 .. 20; the difference of two values is off by their errors over the step, and by h^2 |act'''| / 6 <= 0.01 * 2 / 6)
    mid = slice(801, 1200)
    got, step = _np(b.apb_gated_forward(gu, kind))[:, 0], 0.1
    diff = (got[802:1201] - got[800:1199]) / (2 * step)
    err = np.abs(diff - dgu[mid, 0])
    assert np.all(err[np.abs(x[mid]) > 0.15] <= 0.004 + 1e-4)
    odd = torch.tensor([[np.inf, 1.0], [-np.inf, 1.0], [np.nan, 1.0]], dtype=torch.float32, device="cuda")
    v = b.apb_gated_forward(odd, kind).cpu().numpy()[:, 0]
    d = b.apb_gated_backward(odd, torch.ones(3, 1, device="cuda"), kind).cpu().numpy()
    assert v[0] == np.inf and v[1] == 0 and np.isnan(v[2])
    assert d[0, 0] == 1 and d[1, 0] == 0 and d[0, 1] == np.inf and d[1, 1] == 0 and np.isnan(d[2, 1])


# ------------------------------------------------------------------------------------------ the product

def _projections(x_codes, w_codes, K, N, E, offsets, rows_from=None):
    """G, U and the sums of their terms' magnitudes, in float64."""
    xv, wv = o4.values(*x_codes, K), o4.values(*w_codes, K)
    xv = xv if rows_from is None else xv[rows_from]
    M = xv.shape[0]
    gu, mag = np.zeros((M, 2 * N)), np.zeros((M, 2 * N))
    bounds = [0, M] if offsets is None else offsets
    for e in range(E):
        rows, w = slice(bounds[e], bounds[e + 1]), wv[e * 2 * N:(e + 1) * 2 * N]
        gu[rows], mag[rows] = xv[rows] @ w.T, np.abs(xv[rows]) @ np.abs(w).T
    return gu, mag


def _check_product(y, gu, mag, K, kind, t):
    N = gu.shape[1] // 2
    eps = (K / 16 + 64) * 2.0 ** -23
    g, u, eg, eu = gu[:, :N], gu[:, N:], eps * mag[:, :N], eps * mag[:, N:]
    v, d, ev, _ = _act_error(g, kind)
    near = np.abs(v) + 1.13 * eg                                     # (|act'| <= 1.13)
    _check(_np(y), v * u, (1.13 * eg + ev) * (np.abs(u) + eu) + near * eu + 2.0 ** -23 * np.abs(v * u), t)


def _check_saved(saved, gu, mag, K, M, N, inside):
    """Half a step off, or the whole of one beyond 126.5; the scale is that of the largest value."""
    eps = (K / 16 + 64) * 2.0 ** -23
    codes, scales = o.unpack8(saved.cpu().numpy(), 2 * M, N)
    want = np.concatenate([gu[:, :N], gu[:, N:]])
    err = eps * np.concatenate([mag[:, :N], mag[:, N:]])
    step = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, 1)[:, :N]
    got = o.values8(codes, scales, N)
    tol = np.where(np.abs(want) + err > 126.5 * step, 1.0, 0.5) * step * 1.0001 + err
    assert (np.abs(got - want) <= tol).all()
    assert (codes[:, N:] == 0).all()
    low, high = o.quantize8(np.maximum(np.abs(want) - err, 0))[1], o.quantize8(np.abs(want) + err)[1]
    assert (low <= scales).all() and (scales <= high).all()
    rows = np.concatenate([inside, inside])
    assert (codes[~rows] == 0).all() and (scales[~rows] == 0).all()


@pytest.mark.parametrize("kind,t", [("silu", "bf16"), ("gelu", "f32"), ("relu", "f16")])
@pytest.mark.parametrize("M,N,K,E", [c[:4] for c in gated.PRODUCTS])
def test_gated_gemm(b, M, N, K, E, kind, t):
    x, w = _acts(M + N + K, M, K), (np.random.default_rng(N).standard_normal((max(E, 1) * 2 * N, K)) * K ** -0.5).astype(np.float32)
    xc, wc = o4.quantize(x), o4.quantize(w)
    off = cases.offsets(M, E)
    gu, mag = _projections(xc, wc, K, N, max(E, 1), off)
    a4, w4 = torch.from_numpy(o4.pack(*xc)).cuda(), torch.from_numpy(o4.pack(*wc)).cuda()
    offsets = None if off is None else torch.from_numpy(off).cuda()
    frame = torch.full((M, N + 6), 3.0, dtype=TYPE[t], device="cuda")
    saved = torch.full((b.apb_mx8_bytes(2 * M, N),), 99, dtype=torch.uint8, device="cuda")
    b.apb_mx4_gated_gemm(a4, w4, M, N, K, kind, Y=frame[:, 3:N + 3], offsets=offsets, saved=saved)
    assert bool((frame[:, :3] == 3).all() and (frame[:, N + 3:] == 3).all())
    _check_product(frame[:, 3:N + 3], gu, mag, K, kind, t)
    inside = np.arange(M) < (M if off is None else off[-1])
    _check_saved(saved, gu, mag, K, M, N, inside)
    y = b.apb_mx4_gated_gemm(a4, w4, M, N, K, kind, dtype=TYPE[t], offsets=offsets)      # (few rows: the other kernel)
    _check_product(y, gu, mag, K, kind, t)
    assert torch.equal(y, b.apb_mx4_gated_gemm(a4, w4, M, N, K, kind, dtype=TYPE[t], offsets=offsets))
    assert bool((y[torch.from_numpy(~inside).cuda()] == 0).all())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,N,K,E,k", [(1, 70, 300, 0, 1), (5, 33, 4096, 0, 1), (16, 65, 256, 8, 3), (3, 50, 100, 64, 4), (300, 130, 520, 0, 1),
                                       (90, 66, 300, 4, 2), (900, 515, 200, 6, 2)])
def test_gated_linear(b, T, N, K, E, k, t):
    g = np.random.default_rng(T + N)
    x, v = _in(_acts(T + K, T, K), t)
    w = (g.standard_normal((max(E, 1) * 2 * N, K)) * K ** -0.5).astype(np.float32)
    w4 = b.apb_mx4_quantize(torch.from_numpy(w).cuda())
    rows = off = None
    kw = {}
    if E:
        expert = np.sort(g.integers(0, E, T * k))
        rows = g.integers(0, T, T * k).astype(np.int32)
        off = np.searchsorted(expert, np.arange(E + 1)).astype(np.int32)
        kw = dict(rows_from=torch.from_numpy(rows).cuda(), offsets=torch.from_numpy(off).cuda())
    gu, mag = _projections(o4.quantize(v), o4.quantize(w), K, N, max(E, 1), off, rows)
    y = b.apb_mx4_gated_linear(_wide(x), w4, N, "silu", **kw)
    assert y.dtype == TYPE[t]
    _check_product(y, gu, mag, K, "silu", t)
    M = T * k if E else T
    saved = b.alloc_mx8(2 * M, N)
    y = b.apb_mx4_gated_linear(x, w4, N, "silu", saved=saved, **kw)
    _check_product(y, gu, mag, K, "silu", t)
    _check_saved(saved, gu, mag, K, M, N, np.ones(M, bool))
    scratch = torch.empty(max(b.apb_mx4_gated_linear_scratch_bytes(bool(E), max(E, 1), M, N, K), 1), dtype=torch.uint8, device="cuda")
    assert torch.equal(b.apb_mx4_gated_linear(x, w4, N, "silu", scratch=scratch, **kw), b.apb_mx4_gated_linear(x, w4, N, "silu", **kw))


def test_gated_blocks_of_nan_and_zero(b):
    """A NaN in a row or in a weight reaches exactly the outputs it enters; a row of zeros gives zeros."""
    M, N, K = 40, 50, 300
    x, w = _acts(1, M, K), (np.random.default_rng(2).standard_normal((2 * N, K)) * 0.05).astype(np.float32)
    x[5, 7], x[9] = np.nan, 0.0
    w[11, 3], w[N + 20, 290] = np.inf, np.nan
    saved = b.alloc_mx8(2 * M, N)
    w4 = b.apb_mx4_quantize(torch.from_numpy(w).cuda())
    y = b.apb_mx4_gated_linear(torch.from_numpy(x).cuda(), w4, N, saved=saved).cpu().numpy()
    want = np.zeros((M, N), bool)
    want[5], want[:, 11], want[:, 20] = True, True, True
    assert np.array_equal(np.isnan(y), want)
    assert (y[9][~want[9]] == 0).all()
    back = b.apb_mx8_dequantize(saved, 2 * M, N).cpu().numpy()
    assert np.isnan(back[5]).all() and np.isnan(back[:M, :32]).all() and not np.isnan(back[:M, 32:][np.arange(M) != 5]).any()
    assert np.isnan(back[M:, :32]).all()
    few = b.apb_mx4_gated_linear(torch.from_numpy(x[:10]).cuda(), w4, N).cpu().numpy()
    assert np.array_equal(np.isnan(few), want[:10])


def test_rows_beyond_32_bits(b):
    """Matrices of more than 2^32 bytes and 2^31 elements: their last rows against the same rows by themselves, to the bit."""
    M, N = 70000, 16000
    gu = torch.empty(M, 2 * N, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for at in range(0, M, 10000):
        gu[at:at + 10000] = torch.randn(10000, 2 * N, generator=g, device="cuda").bfloat16()
    dy = gu[:, :N].contiguous()
    saved = b.alloc_mx8(2 * M, N)
    y = b.apb_gated_forward(gu, "silu", saved=saved)
    dgu = b.apb_gated_backward(saved, dy, "silu")
    tail = slice(M - 50, M)
    few = b.alloc_mx8(100, N)
    assert torch.equal(y[tail], b.apb_gated_forward(gu[tail], "silu", saved=few))
    assert torch.equal(dgu[tail], b.apb_gated_backward(few, dy[tail], "silu"))
    del y, dgu, dy
    x8 = b.apb_mx8_quantize(gu)
    back = b.apb_mx8_dequantize(x8, M, 2 * N, torch.bfloat16)
    assert torch.equal(back[tail], b.apb_mx8_dequantize(b.apb_mx8_quantize(gu[tail]), 50, 2 * N, torch.bfloat16))


def test_gated_refusals(b):
    x = torch.zeros(4, 64, device="cuda")
    w4 = b.apb_mx4_quantize(torch.zeros(80, 64, device="cuda"))
    with pytest.raises(ValueError):
        b.apb_mx4_gated_linear(x, w4, 40, "tanh")
    with pytest.raises(ValueError):
        b.apb_mx4_gated_linear(x, w4, 41)
    with pytest.raises(ValueError):
        b.apb_mx4_gated_linear(x, w4, 40, saved=b.alloc_mx8(7, 40))
    with pytest.raises(ValueError):
        b.apb_mx4_gated_linear(x, w4, 40, Y=torch.empty(4, 41, device="cuda"))
    with pytest.raises(ValueError):
        b.apb_mx4_gated_linear(torch.zeros(100, 64, device="cuda"), w4, 40, scratch=torch.empty(5, dtype=torch.uint8, device="cuda"), saved=b.alloc_mx8(200, 40))
    with pytest.raises(ValueError):
        b.apb_gated_forward(torch.zeros(4, 7, device="cuda"))
    with pytest.raises(TypeError):
        b.apb_gated_forward(torch.zeros(4, 8, device="cuda"), Y=torch.empty(4, 4, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        b.apb_gated_backward(torch.zeros(4, 8, device="cuda"), torch.zeros(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        b.apb_gated_backward(b.alloc_mx8(8, 4)[:100], torch.zeros(4, 4, device="cuda"))
    with pytest.raises(TypeError):
        b.apb_gated_backward(torch.zeros(4, 8, device="cuda"), torch.zeros(4, 4, device="cuda"), Y=torch.empty(4, 4, device="cuda", dtype=torch.float16))
    with pytest.raises(TypeError):
        b.apb_mx8_quantize(torch.zeros(4, 8, device="cuda", dtype=torch.float64))
    with pytest.raises(TypeError):
        b.apb_mx8_quantize(torch.zeros(4, 8, device="cuda").t())
