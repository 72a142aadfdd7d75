"""The microscaled 4-bit matrices through the C ABI against the CPU oracle in float64.

Tolerances, fixed before the first run.  Quantization: none, bytes are compared.  Dequantization: the value rounded once.
Products and gradients: 4-bit values, their products and the parts of G are exact, so an error is made only where float32 sums
are rounded.  A sum passes through at most (terms / 16 + 64) additions in a row (matrix instructions chained over at least 16
terms each, a tree of no more than 64 inside one, joins of partial sums), each within 2^-23 of the sum of the magnitudes of the
terms, whether it rounds or cuts off; then one rounding to the output's type."""
import numpy as np
import pytest
import torch

import mx4_tile_cases as cases
from oracle import mx4_oracle as o

pytestmark = pytest.mark.gpu

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {t: torch.finfo(d).eps / 2 for t, d in TYPE.items()}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
PARTS = {"f32": 3, "bf16": 1, "f16": 2}


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2306_08960_amd import binding
    binding.load()
    return binding


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _in(a, t):
    """float array -> GPU tensor of type t, and the same values in float32."""
    x = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPE[t])
    return x.cuda(), x.float().numpy()


def _close(got, want, mag, terms, t, parts=1):
    tol = (parts * terms / 16 + 64) * 2.0 ** -23 * mag + HALF_ULP[t] * 1.001 * (np.abs(want) + 2.0 ** -10 * mag) + TINY[t]
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (worst, got[worst], want[worst], tol[worst])


def _acts(seed, M, K):
    g = np.random.default_rng(seed)
    return (g.standard_normal((M, K)) * np.exp(g.standard_normal(K))).astype(np.float32)


def _weights(seed, rows, K):
    return (np.random.default_rng(seed + 7919).standard_normal((rows, K)) * 0.02).astype(np.float32)


# ------------------------------------------------------------------------------------------ quantization

def _special(M, K):
    """Values where rounding and scales go wrong: midway points, saturation, subnormals, zeros, the extremes."""
    g = np.random.default_rng(M * 10007 + K)
    x = _acts(M + K, M, K)
    mids = np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5, 7, 7.99], np.float32)
    for r in range(0, M, 2):
        x[r] = g.choice(mids, K) * g.choice([-1, 1], K) * np.float32(2.0) ** int(g.integers(-6, 7))
    x[1 % M] = 0
    x[-1, :] *= np.float32(1e-4)
    return x


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 31), (3, 32), (5, 33), (2, 255), (7, 256), (3, 257), (16, 517), (33, 1024), (9, 4096)])
def test_quantize_and_back(b, M, K, t):
    x, v = _in(_special(M, K), t)
    codes, scales = o.quantize(v)
    mx = b.apb_mx4_quantize(x)
    assert np.array_equal(mx.cpu().numpy(), o.pack(codes, scales))
    want = o.values(codes, scales, K)
    for back in ("f32", "bf16", "f16"):
        got = b.apb_mx4_dequantize(mx, M, K, TYPE[back])
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(TYPE[back]))


def test_quantize_extremes(b):
    x = np.zeros((8, 64), np.float32)
    x[0, :40] = 3.4028235e38
    x[1, :4] = 1e-45, -3e-39, 1.1754944e-38, 5e-39
    x[2, 3], x[2, 40] = np.inf, 1.0
    x[3, 3], x[3, 40] = np.nan, -1.0
    x[4, 0], x[4, 1] = -np.inf, 5.0
    x[5, :2] = 1e30, 1e-30
    x[6, :] = -0.0
    codes, scales = o.quantize(x)
    mx = b.apb_mx4_quantize(torch.from_numpy(x).cuda())
    assert np.array_equal(mx.cpu().numpy(), o.pack(codes, scales))
    got = b.apb_mx4_dequantize(mx, 8, 64).cpu().numpy()
    assert np.array_equal(got, o.values(codes, scales, 64).astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_quantize_strides_and_gather(b, t):
    M, K = 70, 300
    x, v = _in(_special(M, K), t)
    want = o.pack(*o.quantize(v))
    wide = torch.full((M, K + 5), 99.0, dtype=TYPE[t], device="cuda")
    wide[:, 3:K + 3] = x
    every = torch.full((2 * M, 3 * K), 99.0, dtype=TYPE[t], device="cuda")
    every[::2, ::3] = x
    for view in (x, wide[:, 3:K + 3], x.t().contiguous().t(), every[::2, ::3]):
        mx = torch.full((b.apb_mx4_bytes(M, K),), 0xa5, dtype=torch.uint8, device="cuda")
        assert np.array_equal(b.apb_mx4_quantize(view, mx=mx).cpu().numpy(), want)
    rows = np.array([5, 5, -1, 69, 0, 70, 2 ** 31 - 1, 3], np.int32)
    there = (rows >= 0) & (rows < M)
    picked = np.where(there[:, None], v[np.where(there, rows, 0)], 0).astype(np.float32)
    for view in (x, x.t().contiguous().t()):
        mx = b.apb_mx4_quantize(view, rows_from=torch.from_numpy(rows).cuda())
        assert np.array_equal(mx.cpu().numpy(), o.pack(*o.quantize(picked)))


def test_dequantize_into_a_wider_matrix(b):
    x, v = _in(_special(6, 70), "f32")
    mx = b.apb_mx4_quantize(x)
    for pad in (1, 2):                                               # rows that start at odd and at even places
        out = torch.full((6, 70 + pad), 7.0, device="cuda")
        b.apb_mx4_dequantize(mx, 6, 70, X=out[:, :70])
        assert np.array_equal(out[:, :70].cpu().numpy(), o.quantized(v).astype(np.float32)) and (out[:, 70:] == 7.0).all()


# ------------------------------------------------------------------------------------------ products

SHAPES = [(1, 1, 1), (1, 33, 40), (2, 64, 256), (3, 100, 300), (15, 129, 512), (16, 200, 513), (17, 48, 1000), (31, 77, 2048),
          (33, 517, 96), (64, 256, 768), (65, 130, 257), (127, 255, 512), (130, 300, 1024), (257, 259, 600), (1, 1000, 4096),
          (300, 513, 4200), (520, 528, 300)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("t,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
def test_linear(b, M, N, K, t, out):
    print(f"[case] mx4 linear {M} {N} {K} {t} {out}", flush=True)
    x, v = _in(_acts(M + N + K, M, K), t)
    wf = _weights(N + K, N, K)
    w4 = b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    want, mag = o.product(o.quantized(v), o.quantized(wf), N)
    guard = torch.full((M + 2, N + 3), 7.0, dtype=TYPE[out], device="cuda")
    y = guard[1:M + 1, :N]
    b.apb_mx4_linear(x, w4, N, Y=y)
    _close(_np(y), want, mag, K, out)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (guard[:, N:] == 7).all()
    y2 = b.apb_mx4_gemm(b.apb_mx4_quantize(x), w4, M, N, K, dtype=TYPE[out])
    _close(_np(y2), want, mag, K, out)
    # exchanged operands: the transposed product
    y3 = b.apb_mx4_gemm(w4, b.apb_mx4_quantize(x), N, M, K, dtype=TYPE[out])
    _close(_np(y3).T, want, mag, K, out)


@pytest.mark.parametrize("M,N,K", [(16, 200, 4096), (12, 70, 5000), (5, 33, 13000)])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_linear_few_long_rows(b, M, N, K, t):
    # rows that fill most of a compute unit's LDS
    print(f"[case] mx4 linear {M} {N} {K} {t}", flush=True)
    x, v = _in(_acts(M + N + K, M, K), t)
    wf = _weights(N + K, N, K)
    w4 = b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    want, mag = o.product(o.quantized(v), o.quantized(wf), N)
    y = b.apb_mx4_linear(x, w4, N)
    _close(_np(y), want, mag, K, t)
    y = b.apb_mx4_gemm(b.apb_mx4_quantize(x), w4, M, N, K, dtype=TYPE[t])
    _close(_np(y), want, mag, K, t)


def _groups(kind, M, E, seed=0):
    g = np.random.default_rng(seed + M + E)
    if kind == "even":
        cut = np.arange(E + 1) * M // E
    elif kind == "one":                                              # one expert has all rows
        cut = np.array([0] * (E // 2 + 1) + [M] * (E - E // 2))
    elif kind == "none":                                             # no row has an expert
        cut = np.zeros(E + 1)
    else:                                                            # ragged, some empty, some rows behind the last
        cut = np.sort(np.concatenate([[0], g.integers(0, M + 1, E)]))
        cut[E // 2] = cut[E // 2 + 1] if E > 1 else cut[E // 2]
        cut = np.minimum(np.sort(cut), max(M - 3, 0))
    return cut.astype(np.int32)


GROUPS = [("even", 8, 4, 64, 256), ("ragged", 37, 5, 100, 300), ("ragged", 1, 3, 33, 70), ("one", 40, 6, 96, 512),
          ("none", 20, 3, 40, 128), ("ragged", 300, 7, 257, 520), ("even", 640, 3, 200, 1024), ("ragged", 200, 130, 48, 256),
          ("ragged", 70, 1, 130, 300), ("one", 600, 4, 300, 768), ("ragged", 900, 2, 520, 300)]


@pytest.mark.parametrize("kind,M,E,N,K", GROUPS)
@pytest.mark.parametrize("t,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_grouped(b, kind, M, E, N, K, t, out):
    print(f"[case] mx4 grouped {kind} {M} {E} {N} {K} {t}", flush=True)
    tokens = M // 2 + 1
    x, v = _in(_acts(M + N + K, tokens, K), t)
    rows = np.random.default_rng(M).integers(0, tokens, M).astype(np.int32)
    off = _groups(kind, M, E)
    wf = _weights(N + K, E * N, K)
    w4 = b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    want, mag = o.product(o.quantized(v)[rows], o.quantized(wf), N, off)
    y = torch.full((M, N), 7.0, dtype=TYPE[out], device="cuda")
    dev = torch.from_numpy(off).cuda()
    b.apb_mx4_linear(x, w4, N, Y=y, rows_from=torch.from_numpy(rows).cuda(), offsets=dev)
    _close(_np(y), want, mag, K, out)
    assert (_np(y)[off[-1]:] == 0).all()
    y2 = torch.full((M, N), 7.0, dtype=TYPE[out], device="cuda")
    b.apb_mx4_gemm(b.apb_mx4_quantize(x, rows_from=torch.from_numpy(rows).cuda()), w4, M, N, K, Y=y2, offsets=dev)
    _close(_np(y2), want, mag, K, out)


@pytest.mark.parametrize("M", [3, 200])
def test_nan_stays_in_its_row(b, M):
    x = _acts(5, M, 300)
    x[1, 290], x[2, 0] = np.nan, np.inf
    w4 = b.apb_mx4_quantize(torch.from_numpy(_weights(5, 70, 300)).cuda())
    for y in (b.apb_mx4_linear(torch.from_numpy(x).cuda(), w4, 70),
              b.apb_mx4_gemm(b.apb_mx4_quantize(torch.from_numpy(x).cuda()), w4, M, 70, 300)):
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
        assert torch.isfinite(y[0]).all() and torch.isfinite(y[3:]).all()


def test_offsets_that_make_no_sense_stay_in_bounds(b):
    M, E, N, K = 50, 4, 40, 300
    x = torch.from_numpy(_acts(1, M, K)).cuda()
    w4 = b.apb_mx4_quantize(torch.from_numpy(_weights(1, E * N, K)).cuda())
    x4 = b.apb_mx4_quantize(x)
    g = torch.randn(M, N, device="cuda")
    for bad in ([0, 60, 10, 2 ** 31 - 1, 50], [-5, -1, 40, 20, 90], [50, 40, 30, 20, 10]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        guard = torch.full((M + 2, N), 7.0, device="cuda")
        b.apb_mx4_linear(x, w4, N, Y=guard[1:-1], offsets=off)
        b.apb_mx4_gemm(x4, w4, M, N, K, Y=guard[1:-1], offsets=off)
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()
        b.apb_mx4_backward_input(g, w4, K, offsets=off)
        b.apb_mx4_backward_weight(g, x4, K, offsets=off)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------ gradients

@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 33, 40), (3, 100, 300), (17, 64, 256), (64, 130, 513), (130, 70, 257),
                                   (200, 300, 520), (333, 257, 130), (520, 300, 300)])
@pytest.mark.parametrize("t,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
def test_gradients(b, M, N, K, t, out):
    print(f"[case] mx4 gradients {M} {N} {K} {t} {out}", flush=True)
    xf, wf = _acts(M + K, M, K), _weights(N + K, N, K)
    g, gv = _in(np.random.default_rng(M * N).standard_normal((M, N)) * 1e-2, t)
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    dx, dw, mx, mw = o.gradients(gv, o.quantized(xf), o.quantized(wf))
    gx, gw = torch.full((M, K + 2), 7.0, dtype=TYPE[out], device="cuda"), torch.full((N, K + 2), 7.0, dtype=TYPE[out], device="cuda")
    b.apb_mx4_backward_input(g, w4, K, dX=gx[:, :K])
    b.apb_mx4_backward_weight(g, x4, K, dW=gw[:, :K])
    _close(_np(gx[:, :K]), dx, mx, N, out, PARTS[t])
    _close(_np(gw[:, :K]), dw, mw, M, out, PARTS[t])
    assert (gx[:, K:] == 7).all() and (gw[:, K:] == 7).all()
    # a gradient whose rows do not start at 16-byte boundaries
    odd = torch.zeros((M, N + 3), dtype=TYPE[t], device="cuda")
    odd[:, 1:N + 1] = g
    _close(_np(b.apb_mx4_backward_input(odd[:, 1:N + 1], w4, K, dtype=TYPE[out])), dx, mx, N, out, PARTS[t])
    _close(_np(b.apb_mx4_backward_weight(odd[:, 1:N + 1], x4, K, dtype=TYPE[out])), dw, mw, M, out, PARTS[t])


@pytest.mark.parametrize("kind,M,E,N,K", GROUPS)
@pytest.mark.parametrize("t,out", [("f32", "f32"), ("bf16", "bf16")])
def test_grouped_gradients(b, kind, M, E, N, K, t, out):
    print(f"[case] mx4 grouped gradients {kind} {M} {E} {N} {K} {t}", flush=True)
    xf, wf, off = _acts(M + K, M, K), _weights(N + K, E * N, K), _groups(kind, M, E)
    g, gv = _in(np.random.default_rng(M * N).standard_normal((M, N)) * 1e-2, t)
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    dx, dw, mx, mw = o.gradients(gv, o.quantized(xf), o.quantized(wf), off)
    dev = torch.from_numpy(off).cuda()
    gx, gw = torch.full((M, K), 7.0, dtype=TYPE[out], device="cuda"), torch.full((E * N, K), 7.0, device="cuda")
    b.apb_mx4_backward_input(g, w4, K, dX=gx, offsets=dev)
    b.apb_mx4_backward_weight(g, x4, K, dW=gw, offsets=dev)
    _close(_np(gx), dx, mx, N, out, PARTS[t])
    _close(_np(gw), dw, mw, M, "f32", PARTS[t])


@pytest.mark.parametrize("M,N,K,E", [(5000, 70, 130, 0), (60, 4100, 70, 0), (2100, 2500, 33, 0), (4096, 512, 40, 3), (9000, 40, 300, 2)])
@pytest.mark.parametrize("t,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_long_sums_shared_by_workgroups(b, M, N, K, E, t, out):
    """Few outputs and long sums: shared through a workspace where there is one, with the same tolerance, and the same bits again."""
    print(f"[case] mx4 long sums {M} {N} {K} {E} {t}", flush=True)
    off = _groups("ragged", M, E) if E else None
    dev = None if off is None else torch.from_numpy(off).cuda()
    xf, wf = _acts(M + K, M, K), _weights(N + K, max(E, 1) * N, K)
    g, gv = _in(np.random.default_rng(M * N).standard_normal((M, N)) * 1e-2, t)
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    dx, dw, mx, mw = o.gradients(gv, o.quantized(xf), o.quantized(wf), off)
    args = (TYPE[t], E > 0, max(E, 1), M, N, K)
    shared = b.apb_mx4_backward_input_workspace_bytes(*args), b.apb_mx4_backward_weight_workspace_bytes(*args)
    assert max(shared) > 0
    longest = M if off is None else int(np.diff(off).max())
    for small in (False, True):
        ws = torch.empty(16, dtype=torch.uint8, device="cuda") if small else None
        gx, gw = torch.full((M, K + 1), 7.0, dtype=TYPE[out], device="cuda"), torch.full((max(E, 1) * N, K + 1), 7.0, dtype=TYPE[out], device="cuda")
        b.apb_mx4_backward_input(g, w4, K, dX=gx[:, :K], offsets=dev, workspace=ws)
        b.apb_mx4_backward_weight(g, x4, K, dW=gw[:, :K], offsets=dev, workspace=ws)
        _close(_np(gx[:, :K]), dx, mx, N, out, PARTS[t])
        _close(_np(gw[:, :K]), dw, mw, longest, out, PARTS[t])
        assert (gx[:, K:] == 7).all() and (gw[:, K:] == 7).all()
        assert torch.equal(b.apb_mx4_backward_input(g, w4, K, dtype=TYPE[out], offsets=dev, workspace=ws), gx[:, :K])
        assert torch.equal(b.apb_mx4_backward_weight(g, x4, K, dtype=TYPE[out], offsets=dev, workspace=ws), gw[:, :K])


@pytest.mark.parametrize("M,N,K,E", [(2500, 4133, 2500, 0), (2570, 1030, 2100, 3)])
def test_gradients_of_large_tiles(b, M, N, K, E):
    """Tiles of 256 a side with ragged edges: whole sums, sums shared by two workgroups, and groups."""
    print(f"[case] mx4 large gradients {M} {N} {K} {E}", flush=True)
    off = np.array([0, 700, 700, M - 2], np.int32) if E else None
    dev = None if off is None else torch.from_numpy(off).cuda()
    xf, wf = _acts(M + K, M, K), _weights(N + K, max(E, 1) * N, K)
    g, gv = _in(np.random.default_rng(M * N).standard_normal((M, N)) * 1e-2, "bf16")
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    dx, dw, mx, mw = o.gradients(gv, o.quantized(xf), o.quantized(wf), off)
    for small in (False, True):
        ws = torch.empty(16, dtype=torch.uint8, device="cuda") if small else None
        gx = torch.full((M, K + 1), 7.0, dtype=torch.bfloat16, device="cuda")
        gw = torch.full((max(E, 1) * N, K + 1), 7.0, device="cuda")
        b.apb_mx4_backward_input(g, w4, K, dX=gx[:, :K], offsets=dev, workspace=ws)
        b.apb_mx4_backward_weight(g, x4, K, dW=gw[:, :K], offsets=dev, workspace=ws)
        _close(_np(gx[:, :K]), dx, mx, N, "bf16", 1)
        _close(_np(gw[:, :K]), dw, mw, M, "f32", 1)
        assert (gx[:, K:] == 7).all() and (gw[:, K:] == 7).all()


def test_gradients_by_differences(b):
    """The product is linear in either operand: <G, Y(X, W1) - Y(X, W2)> = <dW, W1^ - W2^>, and the same for X."""
    M, N, K = 96, 80, 320
    x1, x2, w1, w2 = (torch.from_numpy(a).cuda() for a in (_acts(1, M, K), _acts(2, M, K), _weights(1, N, K), _weights(2, N, K)))
    g = torch.randn(M, N, device="cuda")
    q = {n: b.apb_mx4_quantize(v) for n, v in (("x1", x1), ("x2", x2), ("w1", w1), ("w2", w2))}
    y = lambda x, w: b.apb_mx4_gemm(q[x], q[w], M, N, K).double()
    val = lambda n, rows: b.apb_mx4_dequantize(q[n], rows, K).double()
    left = ((y("x1", "w1") - y("x1", "w2")) * g.double()).sum().item()
    term = b.apb_mx4_backward_weight(g, q["x1"], K).double() * (val("w1", N) - val("w2", N))
    # either side: the errors of its float32 sums, (terms / 16 + 64) * 2^-23 of magnitudes that Cauchy-Schwarz bounds
    scale = g.double().norm().item() * val("x1", M).norm().item() * (val("w1", N).norm() + val("w2", N).norm()).item()
    assert abs(left - term.sum().item()) <= 2 * (3 * K / 16 + 64) * 2.0 ** -23 * scale
    left = ((y("x1", "w1") - y("x2", "w1")) * g.double()).sum().item()
    term = b.apb_mx4_backward_input(g, q["w1"], K).double() * (val("x1", M) - val("x2", M))
    scale = g.double().norm().item() * val("w1", N).norm().item() * (val("x1", M).norm() + val("x2", M).norm()).item()
    assert abs(left - term.sum().item()) <= 2 * (3 * K / 16 + 64) * 2.0 ** -23 * scale


@pytest.mark.parametrize("t", ["f32", "f16"])
def test_every_bit_of_the_gradient_counts(b, t):
    """G times a matrix that holds one 1 per row is G itself, to the last bit of its type."""
    N = 64
    w = torch.zeros(N, N)
    w[torch.arange(N), torch.arange(N)] = 1.0
    w4 = b.apb_mx4_quantize(w.cuda())
    g = (torch.randn(40, N) * torch.exp(torch.randn(40, 1) * (3 if t == "f16" else 20))).to(TYPE[t])
    got = b.apb_mx4_backward_input(g.cuda(), w4, N, dtype=torch.float32)
    assert torch.equal(got.cpu(), g.float())


def test_gradients_near_the_ends_of_float32(b):
    """A float32 gradient from the largest values to the smallest: finite where the result is, exact from 2^-125 on."""
    w = torch.zeros(64, 64)
    w[torch.arange(64), torch.arange(64)] = torch.where(torch.arange(64) % 2 == 0, 1.5, 1.0)
    w4 = b.apb_mx4_quantize(w.cuda())
    rows = torch.tensor([127, 126, 100, -90, -109, -111, -118, -120, -124, -125])
    g = torch.ldexp(1 + torch.randint(0, 2 ** 23, (10, 64), generator=torch.Generator().manual_seed(1)).double() * 2.0 ** -23, rows[:, None].double())
    g[0] = 2.0 ** 127 * (1 + 2.0 ** -7 - 2.0 ** -23)                          # (its last 16 bits are as large as they can be)
    got = b.apb_mx4_backward_input(g.float().cuda(), w4, 64, dtype=torch.float32).cpu()
    assert torch.isfinite(got).all()
    assert torch.equal(got[:, 1::2], g[:, 1::2].float())
    assert ((got.double() - g * w.diagonal().double()).abs() <= 2.0 ** -22 * g.abs()).all()
    small = torch.randint(0, 2 ** 24, (64, 64), generator=torch.Generator().manual_seed(2)).double() * 2.0 ** -149
    got = b.apb_mx4_backward_input(small.float().cuda(), w4, 64, dtype=torch.float32).cpu()
    assert ((got.double() - small)[:, 1::2].abs() <= 2.0 ** -148).all()


def test_gradient_infinities_and_nan(b):
    for t in ("f32", "bf16", "f16"):
        g = torch.ones(40, 64, dtype=TYPE[t])
        g[3, 5], g[4, 6] = float("inf"), float("nan")
        w = torch.ones(64, 64)
        dx = b.apb_mx4_backward_input(g.cuda(), b.apb_mx4_quantize(w.cuda()), 64, dtype=torch.float32).cpu()
        assert (dx[3] == float("inf")).all() and torch.isnan(dx[4]).all()
        assert torch.isfinite(dx[:3]).all() and torch.isfinite(dx[5:]).all()


# ------------------------------------------------------------------------------------------ streams, graphs, repeats

def test_same_bits_again_on_another_stream_and_in_a_graph(b):
    M, E, N, K = 70, 5, 130, 520
    x = torch.from_numpy(_acts(9, M, K)).cuda().bfloat16()
    w4 = b.apb_mx4_quantize(torch.from_numpy(_weights(9, E * N, K)).cuda())
    off = torch.from_numpy(_groups("ragged", M, E)).cuda()
    g = torch.randn(M, N, device="cuda").bfloat16()
    x4, scratch = b.alloc_mx4(M, K), b.alloc_mx4(M, K)
    y, dx, dw = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda"), torch.empty(E * N, K, device="cuda")

    def step(stream=None):
        b.apb_mx4_quantize(x, mx=x4, stream=stream)
        b.apb_mx4_linear(x, w4, N, Y=y, offsets=off, scratch=scratch, stream=stream)
        b.apb_mx4_backward_input(g, w4, K, dX=dx, offsets=off, stream=stream)
        b.apb_mx4_backward_weight(g, x4, K, dW=dw, offsets=off, stream=stream)

    def wipe():
        for t in (y, dx, dw):
            t.fill_(7.0)
        x4.fill_(3)

    step()
    first = [t.clone() for t in (x4, y, dx, dw)]
    same = lambda: all(torch.equal(a, c) for a, c in zip(first, (x4, y, dx, dw)))
    side = torch.cuda.Stream()
    wipe()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        wipe()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        (torch.ones(1000, device="cuda") * 2).sum().item()           # eager work in between


def test_binding_refusals(b):
    x, w4 = torch.zeros(4, 64, device="cuda"), b.alloc_mx4(8, 64)
    with pytest.raises(ValueError):
        b.apb_mx4_linear(x, w4, 9)                                    # weights too small
    with pytest.raises(ValueError):
        b.apb_mx4_linear(x, w4, 8, Y=torch.zeros(4, 9, device="cuda"))
    with pytest.raises(TypeError):
        b.apb_mx4_quantize(torch.zeros(4, 64))                        # not on the GPU
    with pytest.raises(TypeError):
        b.apb_mx4_quantize(x.double())
    with pytest.raises(TypeError):
        b.apb_mx4_linear(x.t(), w4, 8)                                # rows not contiguous
    with pytest.raises(TypeError):
        b.apb_mx4_linear(x, w4, 8, offsets=torch.zeros(2, device="cuda"))
    with pytest.raises(b.ApbError) as e:
        b.alloc_mx4(0, 64)
    assert e.value.code == b.APB_ERR_SHAPE
    with pytest.raises(b.ApbError) as e:
        b.apb_mx4_quantize(x, mx=torch.empty(10000, dtype=torch.uint8, device="cuda")[1:])
    assert e.value.code == b.APB_ERR_ALIGN


def test_new_memory_belongs_to_the_calls_stream(b):
    """Outputs and scratch that a call makes come from its stream's memory: what another stream still works on is not in it."""
    side = torch.cuda.Stream()
    x, w4 = torch.randn(300, 256, device="cuda"), b.apb_mx4_quantize(torch.randn(96, 256, device="cuda"))
    logits = torch.randn(300, 8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    r = b.apb_moe_route(logits, 2, stream=side)
    z = torch.zeros(600, 96, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    made = [b.apb_mx4_quantize(x, stream=side), b.apb_mx4_linear(x, w4, 96, stream=side), *r.values()]
    made += [b.apb_mx4_dequantize(made[0], 300, 256, stream=side), b.apb_mx4_gemm(made[0], w4, 300, 96, 256, stream=side)]
    made += [b.apb_mx4_backward_input(made[1], w4, 256, stream=side), b.apb_mx4_backward_weight(made[1], made[0], 256, stream=side)]
    made += [b.apb_moe_combine(z, r["slot_row"], r["weight"], stream=side), *b.apb_moe_combine_backward(made[1], z, r["slot_row"], r["weight"], stream=side)]
    made.append(b.apb_moe_route_backward(r["expert"], r["weight"], made[-1], 8, stream=side))
    side.synchronize()
    segments = torch.cuda.memory_snapshot()
    for t in made:
        home = [s for s in segments if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
        assert len(home) == 1 and home[0]["stream"] == side.cuda_stream
    assert torch.equal(made[1], b.apb_mx4_linear(x, w4, 96))


def test_no_scratch_is_touched_where_none_is_needed(b):
    """The weights stand in for the scratch of the single kernel: they and the result stay what they are."""
    x, w4 = torch.randn(3, 512, device="cuda"), b.apb_mx4_quantize(torch.randn(70, 512, device="cuda"))
    assert b.apb_mx4_linear_scratch_bytes(False, 1, 3, 70, 512) == 0
    before, scratch = w4.clone(), torch.full((b.apb_mx4_bytes(3, 512),), 0xa5, dtype=torch.uint8, device="cuda")
    assert torch.equal(b.apb_mx4_linear(x, w4, 70), b.apb_mx4_linear(x, w4, 70, scratch=scratch))
    assert torch.equal(w4, before) and (scratch == 0xa5).all()


def test_scratch_of_the_published_size_is_enough(b):
    """As many bytes as apb_mx4_linear_scratch_bytes says: none, or what the 4-bit form takes; one byte less is refused."""
    w4 = b.apb_mx4_quantize(torch.from_numpy(_weights(3, 70, 512)).cuda())
    for M in (3, 200):
        x = torch.from_numpy(_acts(M, M, 512)).cuda()
        need = b.apb_mx4_linear_scratch_bytes(False, 1, M, 70, 512)
        assert (need == 0) == (M == 3)
        want = b.apb_mx4_linear(x, w4, 70)
        assert torch.equal(b.apb_mx4_linear(x, w4, 70, scratch=torch.empty(need, dtype=torch.uint8, device="cuda")), want)
        if need:
            with pytest.raises(ValueError):
                b.apb_mx4_linear(x, w4, 70, scratch=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
        with pytest.raises(TypeError):
            b.apb_mx4_linear(x, w4, 70, scratch=torch.empty(need, device="cuda"))


# ------------------------------------------------------------------------------------------ every tile size

@pytest.mark.parametrize("M,N,K,E,side", cases.PRODUCTS)
def test_products_of_every_tile_size(b, M, N, K, E, side):
    """Ragged products by tiles of 64, 128 and 256 a side, plain and in groups, into every type; what lies around Y stays."""
    print(f"[case] mx4 tiles {M} {N} {K} {E} {side}", flush=True)
    off = cases.offsets(M, E)
    dev = None if off is None else torch.from_numpy(off).cuda()
    xf, wf = _acts(M + N + K, M, K), _weights(N + K, max(E, 1) * N, K)
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    want, mag = o.product(o.quantized(xf), o.quantized(wf), N, off)
    for out in ("f32", "bf16", "f16"):
        guard = torch.full((M + 2, N + 5), 7.0, dtype=TYPE[out], device="cuda")
        y = guard[1:M + 1, 2:N + 2]
        b.apb_mx4_gemm(x4, w4, M, N, K, Y=y, offsets=dev)
        _close(_np(y), want, mag, K, out)
        assert E == 0 or (y[int(off[-1]):] == 0).all()
        y.fill_(7.0)
        assert (guard == 7).all()
        again = b.apb_mx4_linear(torch.from_numpy(xf).cuda(), w4, N, dtype=TYPE[out], offsets=dev)
        assert torch.equal(again, b.apb_mx4_gemm(x4, w4, M, N, K, dtype=TYPE[out], offsets=dev))


@pytest.mark.parametrize("M,N,K,E,side", cases.PRODUCTS)
def test_nan_stays_in_its_row_and_column_for_every_tile_size(b, M, N, K, E, side):
    """A block of NaN or of an infinity on either side makes its row or column of Y NaN and changes no bit of another."""
    print(f"[case] mx4 tiles with nan {M} {N} {K} {E} {side}", flush=True)
    off = cases.offsets(M, E)
    dev = None if off is None else torch.from_numpy(off).cuda()
    last = M if off is None else int(off[-1])
    x, w = torch.from_numpy(_acts(M + N, M, K)).cuda(), torch.from_numpy(_weights(N, max(E, 1) * N, K)).cuda()
    y = b.apb_mx4_linear(x, b.apb_mx4_quantize(w), N, offsets=dev)
    rows, cols = [0, last // 2, last - 1], [0, 3, N - 1]
    x[rows[0], 0], x[rows[1], K - 1], x[rows[2], K // 2] = float("nan"), float("inf"), float("-inf")
    got = b.apb_mx4_linear(x, b.apb_mx4_quantize(w), N, offsets=dev)
    assert torch.isnan(got[rows]).all()
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[rows] = False
    assert torch.equal(got[keep], y[keep]) and torch.isfinite(y).all()
    e = max(E, 1) - 1                                                # (the last expert: it has rows)
    first = 0 if off is None else int(off[e])
    for i, n in enumerate(cols):
        w[e * N + n, i * (K - 1) // 2] = (float("nan"), float("inf"), float("nan"))[i]
    got = b.apb_mx4_linear(x, b.apb_mx4_quantize(w), N, offsets=dev)
    assert torch.isnan(got[first:last][:, cols]).all()
    keep_cols = torch.ones(N, dtype=torch.bool, device="cuda")
    keep_cols[cols] = False
    assert torch.equal(got[keep][:, keep_cols], y[keep][:, keep_cols])
    assert torch.equal(got[:first][keep[:first]], y[:first][keep[:first]]) and (got[last:] == 0).all()


@pytest.mark.parametrize("M,N,K,E,t,plan_x,plan_w", cases.GRADIENTS)
def test_gradients_of_every_tile_size(b, M, N, K, E, t, plan_x, plan_w):
    """Sums of many passes, by every kernel there is; with a workspace and without."""
    print(f"[case] mx4 gradients by tiles {M} {N} {K} {E} {t} {plan_x} {plan_w}", flush=True)
    off = cases.offsets(M, E)
    dev = None if off is None else torch.from_numpy(off).cuda()
    xf, wf = _acts(M + K, M, K), _weights(N + K, max(E, 1) * N, K)
    g, gv = _in(np.random.default_rng(M * N).standard_normal((M, N)) * 1e-2, t)
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    dx, dw, mx, mw = o.gradients(gv, o.quantized(xf), o.quantized(wf), off)
    longest = M if off is None else int(np.diff(off).max())
    for small in (False, True):
        ws = torch.empty(16, dtype=torch.uint8, device="cuda") if small else None
        gx = torch.full((M + 1, K + 3), 7.0, dtype=TYPE[t], device="cuda")
        gw = torch.full((max(E, 1) * N + 1, K + 3), 7.0, device="cuda")
        b.apb_mx4_backward_input(g, w4, K, dX=gx[:M, 1:K + 1], offsets=dev, workspace=ws)
        b.apb_mx4_backward_weight(g, x4, K, dW=gw[:-1, 1:K + 1], offsets=dev, workspace=ws)
        _close(_np(gx[:M, 1:K + 1]), dx, mx, N, t, PARTS[t])
        _close(_np(gw[:-1, 1:K + 1]), dw, mw, longest, "f32", PARTS[t])
        for guard, rows in ((gx, M), (gw, max(E, 1) * N)):
            guard[:rows, 1:K + 1] = 7.0
            assert (guard == 7).all()


def _special_blocks(seed, rows, K):
    """Rows with a block of NaN, of an infinity, of values below 2^-126 (scale code 0) and of the largest (252)."""
    x = _weights(seed, rows, K)
    x[rows // 3, 5], x[rows - 1, 40] = np.nan, -np.inf
    x[rows // 2, 64:96] = np.random.default_rng(seed).choice([-1, 1], 32) * np.float32(2.0) ** -126 * np.linspace(0.01, 0.99, 32, dtype=np.float32)
    x[1, 128:160] = np.random.default_rng(seed).choice([-1, 1], 32) * np.float32(3e38) * np.linspace(0.01, 1, 32, dtype=np.float32)
    scales = o.quantize(x)[1]
    assert scales[rows // 3, 0] == scales[rows - 1, 1] == 255 and scales[rows // 2, 2] == 0 and scales[1, 4] == 252
    return x


@pytest.mark.parametrize("M,N,K,t,plan_x,plan_w", cases.SPECIAL)
def test_gradients_of_special_blocks(b, M, N, K, t, plan_x, plan_w):
    """4-bit matrices with blocks of NaN and of the smallest and largest scales: a sum that meets a NaN is NaN, also where it meets it
    with a zero, and no other.  Sums of values near the end of float32 are rounded to a multiple of 2^-149 in each addition."""
    print(f"[case] mx4 gradients of special blocks {M} {N} {K} {t} {plan_x} {plan_w}", flush=True)
    xf, wf = _special_blocks(M + K, M, K), _special_blocks(N + K, N, K)
    # (the small blocks' columns hold nothing else, so that they are what the sums are made of)
    for a in (xf, wf):
        a[np.arange(len(a)) != len(a) // 2, 64:96] = 0
    raw = np.random.default_rng(M * N).standard_normal((M, N)) * 2.0 ** -6
    raw[0] = 0
    raw[:, 0] = 0
    g, gv = _in(raw, t)
    x4, w4 = b.apb_mx4_quantize(torch.from_numpy(xf).cuda()), b.apb_mx4_quantize(torch.from_numpy(wf).cuda())
    with np.errstate(invalid="ignore"):
        dx, dw, mx, mw = o.gradients(gv, o.quantized(xf), o.quantized(wf))
    got = (_np(b.apb_mx4_backward_input(g, w4, K, dtype=torch.float32)), _np(b.apb_mx4_backward_weight(g, x4, K)))
    for have, want, mag, terms in zip(got, (dx, dw), (mx, mw), (N, M)):
        nan = np.isnan(want)
        assert nan[:, :64].all() and not nan[:, 64:].any()
        assert np.array_equal(np.isnan(have), nan)
        err, tol = np.abs(have - want)[:, 64:], (PARTS[t] * terms / 16 + 64) * (2.0 ** -23 * mag[:, 64:] + 2.0 ** -149)
        assert (err <= tol).all(), (np.unravel_index(np.argmax(err - tol), err.shape), err.max())
        assert np.abs(want[:, 64:96]).max() > 2.0 ** -136 and np.abs(want[:, 128:160]).max() > 2.0 ** 115
