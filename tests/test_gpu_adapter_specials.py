"""Adapters: what NaN, infinities and memory beside the operands may reach, in every type, and the precision that the header promises.

A result that does not depend on a value is compared to the bit with the one where that value is an ordinary number: the same
operations in the same order on the same numbers.

Tolerances of single terms, fixed before the first run.  T is split into three bfloat16 parts for the gradients (2^-24 of a term, or
2^-134 times the other factor where T is below 2^-109), and into two for Y (2^-16, or 2^-134; float16: 2^-22, or 2^-39 of the row's
largest).  Up to five products of such parts are added to sums that are otherwise zero: 2^-23 of the term for each.  Y0 is added with a
rounding of what is left, and Y is rounded once to its type."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2306_08960_amd import binding
    binding.load()
    return binding


def _framed(x, fill):
    """x as a window of a wider matrix of `fill`, with rows of it before and behind."""
    w = torch.full((x.shape[0] + 2, x.shape[1] + 11), fill, dtype=x.dtype, device="cuda")
    w[1:-1, 3:3 + x.shape[1]] = x
    return w[1:-1, 3:3 + x.shape[1]]


def _same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# M, K, N, r: every number of ranks that is held in registers, whole and ragged widths, sums that workgroups share (the last three)
SIZES = [(90, 130, 256, 5), (90, 64, 300, 16), (150, 517, 1000, 20), (70, 96, 130, 50), (70, 200, 384, 64), (90, 40, 300, 100),
         (40, 70, 136, 128), (50, 130, 90, 200), (64, 4096, 70, 9), (40, 20, 5, 3), (2600, 40, 24, 4), (3000, 130, 70, 40), (2600, 64, 136, 100)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K,N,r", SIZES)
def test_foreign_values_reach_nothing(b, M, K, N, r, t):
    """Rows of another adapter, of none and behind the last segment, an adapter of other rows and one of none, and all that lies around
    the operands, hold NaN and infinities."""
    L, dt = 4, TYPE[t]
    g = torch.Generator(device="cuda").manual_seed(M + N + r)
    new = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(dt)
    x, dy, A, B, y0 = new(M, K), new(M, N), new(L, r, K), new(L, r, N), new(M, N)
    cut = [0, M // 5, M // 5 + 1, M // 2, M // 2, M - M // 3, M - 7]
    adapter = [0, 1, 2, 2, 1, -1]                                    # (nobody has adapter 3; the last segment has none)
    which = torch.full((M,), -1, device="cuda")
    for s, a in enumerate(adapter):
        which[cut[s]:cut[s + 1]] = a
    seg = dict(offsets=torch.tensor(cut, dtype=torch.int32).cuda(), adapter=torch.tensor(adapter, dtype=torch.int32).cuda())
    assert (b.apb_adapter_gradient_workspace_bytes(6, L, M, K, r) > 0) == (M > 1000)
    foreign, none, mine = which == 1, which < 0, (which == 0) | (which == 2)
    bad = lambda *shape: torch.where(torch.rand(*shape, generator=g, device="cuda") < 0.5, NAN, INF).to(dt)
    dx, ddy, dA_, dB_, dy0 = x.clone(), dy.clone(), A.clone(), B.clone(), y0.clone()
    for m, width in ((dx, K), (ddy, N)):
        m[foreign | none] = bad(int((foreign | none).sum()), width)
    dy0[foreign] = bad(int(foreign.sum()), N)
    for f in (dA_, dB_):
        f[1], f[3] = bad(*f.shape[1:]), bad(*f.shape[1:])
    scale = torch.tensor([0.5, 1.0, 2.0, 1.0], device="cuda")
    dirty_scale = torch.tensor([0.5, NAN, 2.0, INF], device="cuda")

    T = b.apb_adapter_down(x, A, scale=scale, **seg)
    dT = b.apb_adapter_down(_framed(dx, NAN), dA_, scale=dirty_scale, **seg)
    assert _same(T[:, mine], dT[:, mine]) and bool((dT[:, none] == 0).all())
    y = b.apb_adapter_up(T, B, Y0=y0, **seg)
    out = _framed(torch.zeros(M, N, dtype=dt, device="cuda"), 3.0)
    b.apb_adapter_up(dT, dB_, Y0=_framed(dy0, NAN), Y=out, **seg)
    assert _same(y[mine], out[mine]) and _same(out[none], y0[none])
    inplace = _framed(dy0, NAN)
    b.apb_adapter_up(dT, dB_, Y0=inplace, Y=inplace, **seg)
    assert _same(y[mine], inplace[mine]) and _same(inplace[none], y0[none])

    def gradients(T, x, dy):
        x8 = b.apb_mx8_quantize(x)
        return (b.apb_adapter_gradient(T, x, L, **seg), b.apb_adapter_gradient(T, dy, L, **seg), b.apb_adapter_gradient(T, x8, L, K=K, **seg),
                b.apb_adapter_gradient(T, x, L, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"), **seg))
    for clean, dirty in zip(gradients(T, x, dy), gradients(dT, _framed(dx, INF), _framed(ddy, NAN))):
        assert bool(torch.isfinite(clean).all()) and bool((dirty[3] == 0).all())
        assert _same(clean[0], dirty[0]) and _same(clean[2], dirty[2])


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K,N,r", [s for s in SIZES if s[2] > 32])
def test_a_value_reaches_its_own(b, M, K, N, r, t, value):
    """One value that is not finite: every result that it enters is not, and no other."""
    L, dt = 2, TYPE[t]
    g = torch.Generator(device="cuda").manual_seed(M + r)
    new = lambda *shape: (torch.rand(*shape, generator=g, device="cuda") + 0.5).to(dt)
    x, A, B, y0 = new(M, K), new(L, r, K), new(L, r, N), new(M, N)
    half = M // 2
    seg = dict(offsets=torch.tensor([0, half, M], dtype=torch.int32).cuda(), adapter=torch.tensor([1, 0], dtype=torch.int32).cuda())
    T = torch.rand(1, M, r, generator=g, device="cuda") + 0.5
    odd = lambda m: ~torch.isfinite(m)

    def marked(shape, *at):
        m = torch.zeros(shape, dtype=torch.bool, device="cuda")
        m[at] = True
        return m
    row, rank, col, k = half - 1, r - 1, N - 2, K - 1                # the last row of adapter 1, the last rank
    dx = x.clone()
    dx[row, k] = value
    assert torch.equal(odd(b.apb_adapter_down(dx, A, **seg).sum(0)), marked((M, r), row))
    dA_ = A.clone()
    dA_[1, rank, k] = value
    assert torch.equal(odd(b.apb_adapter_down(x, dA_, **seg).sum(0)), marked((M, r), slice(0, half), rank))
    dB_ = B.clone()
    dB_[1, rank, col] = value
    assert torch.equal(odd(b.apb_adapter_up(T, dB_, Y0=y0, **seg)), marked((M, N), slice(0, half), col))
    dT = T.clone()
    dT[0, row, rank] = value
    assert torch.equal(odd(b.apb_adapter_up(dT, B, Y0=y0, **seg)), marked((M, N), row))
    dy0 = y0.clone()
    dy0[row, col] = value
    assert torch.equal(odd(b.apb_adapter_up(T, B, Y0=dy0, **seg)), marked((M, N), row, col))
    x8 = lambda m: b.apb_mx8_quantize(m)
    first = k // 32 * 32
    for X, at in ((dx, slice(k, k + 1)), (x8(dx), slice(first, K))):
        assert torch.equal(odd(b.apb_adapter_gradient(T, X, L, K=K, **seg)), marked((L, r, K), 1, slice(None), at))
    for X in (x, x8(x)):
        assert torch.equal(odd(b.apb_adapter_gradient(dT, X, L, K=K, **seg)), marked((L, r, K), 1, rank))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16", "mx8"])
@pytest.mark.parametrize("M,K,r", [(40, 130, 5), (300, 64, 20), (70, 517, 50), (2000, 100, 16)])
@pytest.mark.parametrize("small", [False, True])
def test_gradient_keeps_its_bits(b, M, K, r, t, small):
    """An adapter for each row: every sum is one term."""
    g = np.random.default_rng(M + K)
    shrink = 2.0 ** -118 if small else 1.0
    T = (g.standard_normal((1, M, r)) * np.exp2(g.integers(-12, 13, (1, M, r))) * shrink).astype(np.float32)
    x = torch.from_numpy((g.standard_normal((M, K)) * (64.0 if small else 1.0)).astype(np.float32)).cuda().to(TYPE.get(t, torch.float32))
    X = b.apb_mx8_quantize(x) if t == "mx8" else x
    xv = (b.apb_mx8_dequantize(X, M, K) if t == "mx8" else x).double().cpu().numpy()
    got = b.apb_adapter_gradient(torch.from_numpy(T).cuda(), X, M, K=K, offsets=torch.arange(M + 1, dtype=torch.int32, device="cuda"))
    want = T[0].astype(np.float64)[:, :, None] * xv[:, None, :]
    tol = (2.0 ** -24 + 5 * 2.0 ** -23) * np.abs(want) + 2.0 ** -134 * np.abs(xv)[:, None, :] + 2.0 ** -149
    err = np.abs(got.double().cpu().numpy() - want)
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (at, err[at], tol[at], want[at])


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N,r", [(40, 256, 1), (40, 130, 12), (100, 300, 16), (33, 128, 30), (64, 517, 50), (40, 200, 100), (30, 130, 200),
                                   (2100, 8200, 20)])
def test_up_keeps_its_bits(b, M, N, r, t):
    """One rank of each row counts, and Y0 takes away what Y's type can hold of the product: what is left shows the bits below."""
    g = np.random.default_rng(M + N)
    T = np.zeros((1, M, r), np.float32)
    rank = g.integers(0, r, M)
    T[0, np.arange(M), rank] = g.uniform(64, 256, M).astype(np.float32)
    B = torch.from_numpy(g.uniform(0.5, 2.0, (1, r, N)).astype(np.float32)).cuda().to(TYPE[t])
    term = T[0, np.arange(M), rank].astype(np.float64)[:, None] * B[0].double().cpu().numpy()[rank]
    y0 = torch.from_numpy(-term).cuda().to(TYPE[t])
    got = b.apb_adapter_up(torch.from_numpy(T).cuda(), B, Y0=y0, adapter=torch.zeros(1, dtype=torch.int32, device="cuda")).double().cpu().numpy()
    want = term + y0.double().cpu().numpy()
    half = torch.finfo(TYPE[t]).eps / 2
    tol = ({"f32": 0.0, "bf16": 2.0 ** -16, "f16": 2.0 ** -22}[t] + 2 * 2.0 ** -23) * np.abs(term)
    tol = tol + (half + 2.0 ** -23) * (np.abs(want) + tol) + (2.0 ** -25 if t == "f16" else 0.0)
    err = np.abs(got - want)
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (at, err[at], tol[at], want[at])


# L adapters, S segments, M rows, K, r
@pytest.mark.parametrize("L,S,M,K,r", [(1, 3, 5000, 64, 4), (3, 9, 6000, 130, 20), (9, 40, 9000, 64, 16), (70, 200, 20000, 64, 4), (300, 30, 20000, 100, 5),
                                       (1500, 5, 9000, 64, 4), (2000, 4096, 30000, 64, 3), (4096, 4096, 40000, 40, 2), (8, 64, 40000, 4100, 9),
                                       (20, 65, 40000, 2000, 40)])
@pytest.mark.parametrize("spread", [True, False])
def test_slices_of_many_adapters(b, L, S, M, K, r, spread):
    """Adapters whose rows workgroups share, in segments wherever they are, evenly or most of them one adapter's.  Whole numbers below
    2^24 all the way: every order of the sums gives the same."""
    g = np.random.default_rng(L + S)
    cut = np.sort(g.integers(0, M - 50, S + 1)) if spread else np.concatenate([np.sort(g.integers(0, M // 5, S)), [M - 50]])
    cut[0] = 0
    which = g.integers(-1, L, S)
    which[-1] = L - 1 if L % 2 else L // 2
    seg = dict(offsets=torch.from_numpy(cut.astype(np.int32)).cuda(), adapter=torch.from_numpy(which.astype(np.int32)).cuda())
    row = torch.full((M,), -1, dtype=torch.long)
    for s in range(S):
        row[cut[s]:cut[s + 1]] = int(which[s])
    T = torch.from_numpy(g.integers(-8, 9, (1, M, r)).astype(np.float32)).cuda()
    x = torch.from_numpy(g.integers(-8, 9, (M, K)).astype(np.float32)).cuda().bfloat16()
    need = b.apb_adapter_gradient_workspace_bytes(S, L, M, K, r)
    assert need > 0 and 64 * 50000 < 1 << 24
    want = torch.zeros(L, r, K, dtype=torch.float64)
    for a in set(row.tolist()) - {-1}:
        mine = (row == a).nonzero().flatten().cuda()
        want[a] = (T[0, mine].double().t().contiguous() @ x[mine].double()).cpu()
    for X, k in ((x, None), (b.apb_mx8_quantize(x), K), (x.float(), None)):
        got = b.apb_adapter_gradient(T, X, L, K=k, workspace=torch.full((need,), 0xff, dtype=torch.uint8, device="cuda"), **seg)
        assert torch.equal(got.cpu().double(), want)
    none = b.apb_adapter_gradient(T, x, L, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"), **seg)
    assert torch.equal(none.cpu().double(), want)
