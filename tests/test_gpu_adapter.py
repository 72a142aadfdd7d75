"""Low-rank adapters through the C ABI against the oracle in float64.

Tolerances, fixed before the first run.  Products of 16-bit values are exact, those of float32 and the sums are rounded to float32: a
sum of n terms passes through at most n / 4 + 64 additions or products in a row (matrix instructions chained over at least four
terms each, joins of partial sums), each within 2^-23 of the sum of the magnitudes.  T is multiplied as it is or as two bfloat16
parts (2^-16 of its terms, where Y is rounded to 16 bits anyway); outputs are rounded once to their type."""
import numpy as np
import pytest
import torch

import adapter_cases as cases
from oracle import block_oracle as o

pytestmark = pytest.mark.gpu

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {t: torch.finfo(d).eps / 2 for t, d in TYPE.items()}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
PARTS = {"f32": 0.0, "bf16": 2.0 ** -16, "f16": 2.0 ** -16}


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
    return x.cuda(), x.double().numpy()


def _check(got, want, tol, t):
    tol = tol + HALF_ULP[t] * 1.001 * (np.abs(want) + tol) + TINY[t]
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (at, got[at], want[at], tol[at])


def _sum(n):
    return (n / 4 + 64) * 2.0 ** -23


def _wide(x, extra=5, at=3, fill=99.0):
    w = torch.full((x.shape[0], x.shape[1] + extra), fill, dtype=x.dtype, device="cuda")
    w[:, at:at + x.shape[1]] = x
    return w[:, at:at + x.shape[1]]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K,N,r,L,kind", cases.CASES)
def test_adapter_forward_and_gradients(b, M, K, N, r, L, kind, t):
    g = np.random.default_rng(M * 31 + K + r)
    x, xv = _in(g.standard_normal((M, K)) * np.exp(g.standard_normal(K) * 0.5), t)
    A, Av = _in(g.standard_normal((L, r, K)) * K ** -0.5, t)
    B, Bv = _in(g.standard_normal((L, r, N)) * r ** -0.5, t)
    y0, y0v = _in(g.standard_normal((M, N)), t)
    dy, dyv = _in(g.standard_normal((M, N)) * 0.1, t)
    scale = torch.from_numpy(g.uniform(0.5, 2.0, L).astype(np.float32))
    sv = scale.double().numpy()
    off, adapter = cases.segments(kind, M, L, r)
    which = o.rows_by_adapter(off, adapter, M, L)
    if kind == "all" and adapter is not None:
        which[:] = adapter[0]
    seg = dict(offsets=None if off is None else torch.from_numpy(off).cuda(), adapter=None if adapter is None else torch.from_numpy(adapter).cuda())
    S = 1 if off is None else len(off) - 1

    T = b.apb_adapter_down(_wide(x), A, scale=scale.cuda(), **seg)
    assert tuple(T.shape) == (b.apb_adapter_parts(S, M, K, r), M, r)
    want, mag = o.down(xv, Av, which, sv)
    eT = _sum(K) * mag
    _check(_np(T).sum(0), want, eT, "f32")
    assert bool((T[:, torch.from_numpy(which < 0).cuda()] == 0).all())
    assert torch.equal(T, b.apb_adapter_down(x, A, scale=scale.cuda(), **seg))

    # from here on T is what the kernel left, its parts added up in float32
    Tv = np.zeros((M, r), np.float32)
    for p in T.cpu().numpy():
        Tv = Tv + p
    Tv = Tv.astype(np.float64)
    add, mag = o.up(Tv, Bv, which), o.up(np.abs(Tv), np.abs(Bv), which)
    tol = (_sum(r) + PARTS[t]) * mag + 2.0 ** -23 * np.abs(y0v)
    frame = torch.full((M, N + 6), 3.0, dtype=TYPE[t], device="cuda")
    b.apb_adapter_up(T, B, Y0=_wide(y0), Y=frame[:, 3:N + 3], **seg)
    assert bool((frame[:, :3] == 3).all() and (frame[:, N + 3:] == 3).all())
    _check(_np(frame[:, 3:N + 3]), y0v + add, tol, t)
    none = torch.from_numpy(which < 0).cuda()
    assert torch.equal(frame[:, 3:N + 3][none], y0[none])
    inplace = y0.clone()
    b.apb_adapter_up(T, B, Y0=inplace, Y=inplace, **seg)
    assert torch.equal(inplace, frame[:, 3:N + 3])
    alone = b.apb_adapter_up(T, B, **seg)
    _check(_np(alone), add, (_sum(r) + PARTS[t]) * mag, t)
    assert bool((alone[none] == 0).all())

    # gradients: dT by the same kernel, dA and dB
    dT = b.apb_adapter_down(dy, B, scale=scale.cuda(), **seg)
    want, mag = o.down(dyv, Bv, which, sv)
    _check(_np(dT).sum(0), want, _sum(N) * mag, "f32")
    for Z, Zv, width in ((x, xv, K), (dy, dyv, N)):
        want, mag = o.gradient(Tv, Zv, which, L), o.gradient(np.abs(Tv), np.abs(Zv), which, L)
        got = b.apb_adapter_gradient(T, _wide(Z), L, **seg)
        assert tuple(got.shape) == (L, r, width)
        _check(_np(got), want, _sum(M) * mag, "f32")
        assert torch.equal(got, b.apb_adapter_gradient(T, Z, L, **seg))
        short = torch.empty(4, dtype=torch.uint8, device="cuda")         # (no room: sums are not shared)
        _check(_np(b.apb_adapter_gradient(T, Z, L, workspace=short, **seg)), want, _sum(M) * mag, "f32")
    x8 = b.apb_mx8_quantize(x)
    kept = o.values8(*o.quantize8(xv.astype(np.float32)), K)
    want, mag = o.gradient(Tv, kept, which, L), o.gradient(np.abs(Tv), np.abs(kept), which, L)
    _check(_np(b.apb_adapter_gradient(T, x8, L, K=K, **seg)), want, _sum(M) * mag, "f32")


def test_gradient_against_differences(b):
    """The loss <Y, dY> is linear in each factor and in X: a step of any size gives its derivative, up to float32's roundings."""
    g = np.random.default_rng(5)
    M, K, N, r, L = 50, 40, 30, 4, 3
    x, A, B, dy = (torch.from_numpy(g.integers(-4, 5, s).astype(np.float32)).cuda() for s in ((M, K), (L, r, K), (L, r, N), (M, N)))
    off, adapter = torch.tensor([0, 7, 7, 30, 45], dtype=torch.int32).cuda(), torch.tensor([2, 0, 1, 2], dtype=torch.int32).cuda()
    seg, scale = dict(offsets=off, adapter=adapter), torch.tensor([0.5, 2.0, 1.0]).cuda()
    loss = lambda x, A, B: (b.apb_adapter_up(b.apb_adapter_down(x, A, scale=scale, **seg), B, **seg).double() * dy.double()).sum().item()
    T, dT = b.apb_adapter_down(x, A, scale=scale, **seg), b.apb_adapter_down(dy, B, scale=scale, **seg)
    grads = dict(x=b.apb_adapter_up(dT, A, **seg), A=b.apb_adapter_gradient(dT, x, L, **seg), B=b.apb_adapter_gradient(T, dy, L, **seg))
    base = dict(x=x, A=A, B=B)
    l0 = loss(**base)
    for name, grad in grads.items():
        for at in [tuple(int(g.integers(0, n)) for n in grad.shape) for _ in range(12)]:
            p = base[name].clone()
            p[at] += 1
            assert loss(**{**base, name: p}) - l0 == grad[at].item()      # (whole numbers below 2^24 all the way: exact)


def test_values_outside_stay_outside(b):
    """NaN and infinities in rows, ranks and adapters that do not take part reach nothing."""
    M, K, N, r, L = 40, 100, 90, 5, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, K, generator=g, device="cuda")
    A, B = torch.randn(L, r, K, generator=g, device="cuda"), torch.randn(L, r, N, generator=g, device="cuda")
    y0 = torch.randn(M, N, generator=g, device="cuda")
    off, adapter = torch.tensor([0, 10, 25, 32], dtype=torch.int32).cuda(), torch.tensor([0, -1, 2], dtype=torch.int32).cuda()
    seg = dict(offsets=off, adapter=adapter)
    clean = b.apb_adapter_up(b.apb_adapter_down(x, A, **seg), B, Y0=y0, **seg)
    dirty = x.clone()
    dirty[10:25] = float("nan")
    dirty[32:] = float("inf")
    A[1], B[1] = float("nan"), float("inf")
    T = b.apb_adapter_down(dirty, A, **seg)
    assert torch.equal(b.apb_adapter_up(T, B, Y0=y0, **seg), clean)
    dA = b.apb_adapter_gradient(T, dirty, L, **seg)
    assert bool(torch.isfinite(dA).all()) and bool((dA[1] == 0).all())
    B[0, 4, 7] = float("inf")                                        # a last rank's infinity: that column of adapter 0's rows alone
    y = b.apb_adapter_up(T, B, Y0=y0, **seg)
    bad = ~torch.isfinite(y)
    assert bool(bad[:10, 7].all()) and int(bad.sum()) == 10 and not bool(torch.isnan(y).any())
    dirty[3, 50] = float("nan")
    T = b.apb_adapter_down(dirty, A, **seg)
    rows = torch.isnan(T).any(2).any(0)
    assert rows.nonzero().flatten().tolist() == [3]


def test_rows_beyond_32_bits(b):
    """X and Y of more than 2^32 bytes and 2^31 elements: the last segment, its gradients too, against the oracle."""
    M, K, r, L, tail = 70000, 32000, 8, 2, 300
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    x[:1000] = 1.0
    x[M - tail:] = torch.randn(tail, K, generator=g, device="cuda").bfloat16()
    A = (torch.randn(L, r, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    seg = dict(offsets=torch.tensor([0, M - tail, M], dtype=torch.int32).cuda(), adapter=torch.tensor([0, 1], dtype=torch.int32).cuda())
    T = b.apb_adapter_down(x, A, **seg)
    xv, Av = _np(x[M - tail:]), _np(A)
    which = np.ones(tail, int)
    want, mag = o.down(xv, Av, which)
    _check(_np(T).sum(0)[M - tail:], want, _sum(K) * mag, "f32")
    Tv = _np(T).sum(0)[M - tail:]
    y = b.apb_adapter_up(T, A, Y0=x, **seg)
    _check(_np(y[M - tail:]), xv + o.up(Tv, Av, which), (_sum(r) + PARTS["bf16"]) * o.up(np.abs(Tv), np.abs(Av), which) + 2.0 ** -23 * np.abs(xv), "bf16")
    del y
    dA = b.apb_adapter_gradient(T, x, L, **seg)
    x8 = b.apb_mx8_quantize(x)
    d8 = b.apb_adapter_gradient(T, x8, L, K=K, **seg)
    for got, v in ((dA, xv), (d8, o.values8(*o.quantize8(xv.astype(np.float32)), K))):
        _check(_np(got[1]), o.gradient(Tv, v, which, L)[1], _sum(tail) * o.gradient(np.abs(Tv), np.abs(v), which, L)[1], "f32")


def test_odd_offsets_are_survived(b):
    """Offsets that the documentation leaves without a result: nothing is read or written out of range."""
    M, K, N, r, L = 64, 96, 80, 4, 2
    x, A, B = torch.ones(M, K, device="cuda"), torch.ones(L, r, K, device="cuda"), torch.ones(L, r, N, device="cuda")
    guard = torch.full((M + 2, N), 5.0, device="cuda")
    for off in ([0, 200, 300], [0, -5, 64], [50, 20, 10], [2 ** 31 - 1, -2 ** 31, 7]):
        seg = dict(offsets=torch.tensor(off, dtype=torch.int32).cuda(), adapter=torch.tensor([7, 1], dtype=torch.int32).cuda())
        T = b.apb_adapter_down(x, A, **seg)
        b.apb_adapter_up(T, B, Y=guard[1:M + 1], **seg)
        b.apb_adapter_gradient(T, x, L, **seg)
        torch.cuda.synchronize()
        assert bool((guard[0] == 5).all() and (guard[M + 1] == 5).all())


def test_adapter_refusals(b):
    x, A, B = torch.zeros(4, 64, device="cuda"), torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 3, 40, device="cuda")
    off, ad = torch.tensor([0, 4], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    T = b.apb_adapter_down(x, A, off, ad)
    for call in (lambda: b.apb_adapter_down(x, A[:, :, :60].contiguous(), off, ad), lambda: b.apb_adapter_down(x, A[0], off, ad),
                 lambda: b.apb_adapter_down(x, A, off, torch.zeros(2, dtype=torch.int32).cuda()),
                 lambda: b.apb_adapter_down(x, A, off, ad, T=torch.empty(2, 4, 3, device="cuda")),
                 lambda: b.apb_adapter_down(x, A, off, ad, scale=torch.ones(3, device="cuda")),
                 lambda: b.apb_adapter_up(T, B[:, :2].contiguous(), offsets=off, adapter=ad), lambda: b.apb_adapter_up(T[0], B, offsets=off, adapter=ad),
                 lambda: b.apb_adapter_up(T, B, Y0=torch.zeros(4, 41, device="cuda"), offsets=off, adapter=ad),
                 lambda: b.apb_adapter_gradient(T, torch.zeros(5, 64, device="cuda"), 2, offsets=off, adapter=ad),
                 lambda: b.apb_adapter_gradient(T, b.apb_mx8_quantize(x), 2, offsets=off, adapter=ad),
                 lambda: b.apb_adapter_gradient(T, x, 2, offsets=off, adapter=ad, dA=torch.empty(2, 3, 63, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: b.apb_adapter_down(x, A.half(), off, ad), lambda: b.apb_adapter_down(x, A.transpose(1, 2).contiguous().transpose(1, 2), off, ad),
                 lambda: b.apb_adapter_up(T.double(), B, offsets=off, adapter=ad),
                 lambda: b.apb_adapter_up(T, B, Y=torch.empty(4, 40, device="cuda", dtype=torch.float16), offsets=off, adapter=ad)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: b.apb_adapter_down(x, A), lambda: b.apb_adapter_gradient(T, x, 0, offsets=off, adapter=ad),
                 lambda: b.apb_adapter_down(x, torch.zeros(1, 257, 64, device="cuda"))):
        with pytest.raises(b.ApbError):
            call()
