"""Routing tokens to experts and joining their results, through the C ABI against the CPU oracle in float64.

Tolerances, fixed before the first run.  Whole numbers: none.  Softmax weights: the exponential (2 ulp), a sum of up to 32 terms,
a quotient: 64 * 2^-24 relative.  Gradient of the logits: the same for each factor, sums of 32 terms: 128 * 2^-24 of the sum of
the magnitudes.  Combine: k multiply-adds, (k + 1) * 2^-24 of the magnitudes; dweight: N of them.  Then one rounding."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as o

pytestmark = pytest.mark.gpu

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {t: torch.finfo(d).eps / 2 for t, d in TYPE.items()}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
U = 2.0 ** -24


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


def _logits(T, E, kind):
    g = np.random.default_rng(T * 1009 + E)
    z = g.standard_normal((T, E)) * 2
    if kind == "masked":
        z[g.random((T, E)) < 0.3] = -np.inf
        z[g.random(T) < 0.2] = -np.inf
        z[0] = -np.inf
        z[T // 2, : E // 2] = np.nan
        z[-1] = np.finfo(np.float32).min                             # the type's lowest value can be taken
    if kind == "ties":
        z = np.round(z)
    if kind == "equal":
        z[:] = -0.0
        z[:, ::2] = 0.0
    if kind == "far":
        z *= 100
    return z


@pytest.mark.parametrize("T,E,k,kind,t", [
    (1, 1, 1, "plain", "f32"), (1, 64, 4, "plain", "f32"), (3, 5, 5, "masked", "bf16"), (63, 64, 8, "ties", "bf16"), (64, 8, 2, "ties", "f16"),
    (65, 100, 7, "masked", "f32"), (130, 128, 8, "ties", "f32"), (200, 130, 3, "masked", "f16"), (300, 256, 32, "ties", "bf16"),
    (70, 257, 4, "plain", "f32"), (129, 1024, 6, "masked", "f32"), (500, 3, 2, "masked", "f32"), (1000, 16, 1, "far", "bf16"),
    (64, 32, 32, "masked", "f32"), (64, 1024, 32, "ties", "bf16"), (66, 40, 2, "equal", "f32"), (4200, 12, 3, "masked", "bf16")])
def test_route(b, T, E, k, kind, t):
    print(f"[case] route {T} {E} {k} {kind} {t}", flush=True)
    z, v = _in(_logits(T, E, kind), t)
    if kind == "equal":
        v = np.zeros_like(v)                                         # -0 and 0 are equal: the lowest index goes first
    want = o.route(v, k)
    wide = torch.full((T, E + 3), 50.0, dtype=TYPE[t], device="cuda")
    wide[:, 1:E + 1] = z
    for logits in (z, wide[:, 1:E + 1]):
        got = b.apb_moe_route(logits, k)
        for name in ("expert", "offsets", "row_token", "slot_row"):
            assert np.array_equal(got[name].cpu().numpy(), want[name]), name
        err = np.abs(_np(got["weight"]) - want["weight"])
        assert (err <= 64 * U * want["weight"] + 2.0 ** -126).all()
    d, dv = _in(np.random.default_rng(T).standard_normal((T, k)), "f32")
    w = _np(got["weight"])
    ref = o.route_backward(want["expert"], w, dv, E)
    dl = b.apb_moe_route_backward(got["expert"], got["weight"], d, E, TYPE[t])
    mag = o.route_backward(want["expert"], w, np.zeros_like(dv), E) * 0
    for j in range(k):
        ok = want["expert"][:, j] >= 0
        mag[ok, want["expert"][ok, j]] = (w * (np.abs(dv) + (w * np.abs(dv)).sum(1, keepdims=True)))[ok, j]
    assert (np.abs(_np(dl) - ref) <= 128 * U * mag + HALF_ULP[t] * 1.001 * (np.abs(ref) + 128 * U * mag) + TINY[t]).all()
    assert (_np(dl)[mag == 0] == 0).all()


def test_route_weights_by_differences(b):
    """Central differences of the weights, h = 2^-7 and 2^-8 combined to cancel the h^2 term: what is left is h^4 times a fifth
    derivative (below 1e-8) and the weights' 64 * 2^-24 divided by h."""
    T, E, k, h = 40, 24, 4, 2.0 ** -7
    z = torch.randn(T, E, device="cuda")
    z = torch.round(z * 64) / 64 + torch.arange(E, device="cuda") / 2048          # no two within a step of each other
    d = torch.randn(T, k, device="cuda")
    r = b.apb_moe_route(z, k)
    grad = b.apb_moe_route_backward(r["expert"], r["weight"], d, E).double()
    for j in range(k):
        diff = []
        for s in (h / 128, h / 256):
            hi, lo = z.double(), z.double()
            step = torch.zeros_like(hi).scatter_(1, r["expert"][:, j:j + 1].long(), s)
            f = lambda y: (torch.softmax(y.gather(1, r["expert"].long()), 1) * d.double()).sum(1)
            diff.append((f(hi + step) - f(lo - step)) / (2 * s))
        want = (4 * diff[1] - diff[0]) / 3
        got = grad.gather(1, r["expert"][:, j:j + 1].long())[:, 0]
        assert ((got - want).abs() <= 1e-8 + 256 * U * d.abs().sum(1).double()).all()


@pytest.mark.parametrize("T,E,k,kind,t", [
    (1, 128, 8, "masked", "bf16"), (2, 100, 32, "ties", "f32"), (15, 64, 4, "masked", "f16"), (16, 256, 8, "ties", "bf16"),
    (17, 256, 8, "ties", "bf16"), (16, 512, 4, "masked", "f32"), (80, 512, 32, "ties", "bf16"), (300, 400, 8, "masked", "f32")])
def test_route_few_tokens_and_many_experts(b, T, E, k, kind, t):
    test_route(b, T, E, k, kind, t)


@pytest.mark.parametrize("T,k,N,t", [(1, 1, 1, "f32"), (1, 4, 4096, "bf16"), (3, 2, 7, "f16"), (17, 8, 100, "bf16"), (40, 3, 517, "f32"),
                                     (65, 32, 40, "f16"), (9, 4, 2056, "bf16"), (5, 1, 8192, "f32"), (130, 4, 256, "bf16")])
def test_combine(b, T, k, N, t):
    print(f"[case] combine {T} {k} {N} {t}", flush=True)
    g = np.random.default_rng(T * N + k)
    z, zv = _in(g.standard_normal((T * k, N)), t)
    dy, dyv = _in(g.standard_normal((T, N)), t)
    row = g.permutation(T * k).astype(np.int32).reshape(T, k)
    w = g.random((T, k)).astype(np.float32)
    w[g.random((T, k)) < 0.2] = 0.0
    rd, wd = torch.from_numpy(row).cuda(), torch.from_numpy(w).cuda()
    for weight, dev in ((w, wd), (np.ones_like(w), None)):
        y, mag = o.combine(zv, row, weight), o.combine(np.abs(zv), row, weight)
        dz, dw = o.combine_backward(dyv, zv, row, weight)
        dmag = o.combine_backward(np.abs(dyv), np.abs(zv), row, weight)[1]
        for pad in (0, 1):                                           # rows that do not start at 16-byte boundaries
            wide = lambda a, fill: torch.nn.functional.pad(a, (0, pad), value=fill)[:, :N]
            gy = torch.full((T, N + pad), 7.0, dtype=TYPE[t], device="cuda")
            gz = torch.full((T * k, N + pad), 7.0, dtype=TYPE[t], device="cuda")
            b.apb_moe_combine(wide(z, 7.0), rd, dev, Y=gy[:, :N])
            assert (np.abs(_np(gy[:, :N]) - y) <= (k + 1) * U * mag + HALF_ULP[t] * 1.001 * (np.abs(y) + mag * 2.0 ** -10) + TINY[t]).all()
            _, gw = b.apb_moe_combine_backward(wide(dy, 7.0), wide(z, 7.0), rd, dev, dZ=gz[:, :N])
            assert (np.abs(_np(gz[:, :N]) - dz) <= HALF_ULP[t] * 1.001 * np.abs(dz) + U * np.abs(dz) + TINY[t]).all()
            assert (np.abs(_np(gw) - dw) <= (N + 1) * U * dmag).all()
            assert (gy[:, N:] == 7).all() and (gz[:, N:] == 7).all()
        only, none = b.apb_moe_combine_backward(dy, None, rd, dev)
        assert none is None and torch.equal(only, gz[:, :N].contiguous())


@pytest.mark.parametrize("N,t", [(8192, "bf16"), (8190, "f16"), (4099, "f32")])
def test_combine_beyond_the_caches(b, N, t):
    """Rows larger than the caches are read another way: to the bit what their quarters give, which are not."""
    print(f"[case] large combine {N} {t}", flush=True)
    T, k, q = 2100, 4, 525
    z, dy = torch.randn(T * k, N, device="cuda").to(TYPE[t]), torch.randn(T, N, device="cuda").to(TYPE[t])
    row = torch.cat([torch.randperm(q * k, device="cuda").int().view(q, k) for _ in range(4)])        # within its quarter's rows
    far = row + torch.arange(4, device="cuda", dtype=torch.int32).repeat_interleave(q)[:, None] * (q * k)
    w = torch.rand(T, k, device="cuda")
    y, (dz, dw) = b.apb_moe_combine(z, far, w), b.apb_moe_combine_backward(dy, z, far, w)
    for c in range(4):
        rows, tokens = slice(c * q * k, (c + 1) * q * k), slice(c * q, (c + 1) * q)
        assert torch.equal(y[tokens], b.apb_moe_combine(z[rows], row[tokens], w[tokens]))
        dz_c, dw_c = b.apb_moe_combine_backward(dy[tokens], z[rows], row[tokens], w[tokens])
        assert torch.equal(dz[rows], dz_c) and torch.equal(dw[tokens], dw_c)


def test_slots_of_weight_zero_add_nothing(b):
    z = torch.ones(6, 40, device="cuda")
    z[2], z[5] = float("nan"), float("inf")
    row = torch.tensor([[0, 2], [5, 1], [3, 4]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[1.0, 0.0], [0.0, 2.0], [0.5, 0.5]], device="cuda")
    assert torch.equal(b.apb_moe_combine(z, row, w), torch.tensor([[1.0], [2.0], [1.0]], device="cuda").expand(3, 40))
    dy = torch.full((3, 40), float("inf"), device="cuda")
    dz, _ = b.apb_moe_combine_backward(dy, z, row, w)
    assert (dz[2] == 0).all() and (dz[5] == 0).all() and (dz[0] == float("inf")).all()


def test_rows_out_of_range_are_zeros(b):
    z = torch.ones(4, 40, device="cuda")
    row = torch.tensor([[0, -1], [4, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    y = b.apb_moe_combine(z, row)
    assert (y[0] == 1).all() and (y[1] == 0).all()
    guard = torch.full((6, 40), 7.0, device="cuda")
    _, dw = b.apb_moe_combine_backward(torch.ones(2, 40, device="cuda"), z, row, dZ=guard[1:5])
    assert (guard[1] == 1).all() and (guard[0] == 7).all() and (guard[2:] == 7).all()
    assert dw.tolist() == [[40.0, 0.0], [0.0, 0.0]]
    bad = torch.tensor([[7, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")          # experts that are not there
    dl = b.apb_moe_route_backward(bad, torch.ones(1, 2, device="cuda"), torch.ones(1, 2, device="cuda"), 7)
    assert (dl == 0).all()


def test_graph_replays(b):
    T, E, k, N = 200, 20, 4, 96
    z, ws = torch.randn(T, E, device="cuda"), b.alloc_moe_workspace(T, E, k)
    rows, dy, d = torch.randn(T * k, N, device="cuda"), torch.randn(T, N, device="cuda"), torch.randn(T, k, device="cuda")

    def step():
        r = b.apb_moe_route(z, k, workspace=ws)
        out = [*r.values(), b.apb_moe_route_backward(r["expert"], r["weight"], d, E),
               b.apb_moe_combine(rows, r["slot_row"], r["weight"]), *b.apb_moe_combine_backward(dy, rows, r["slot_row"], r["weight"])]
        return out

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        z.copy_(torch.randn(T, E, device="cuda"))
        ws.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, step()))


def test_refusals(b):
    z = torch.zeros(4, 8, device="cuda")
    for k in (0, 9):
        with pytest.raises(b.ApbError) as e:
            b.apb_moe_route(z, k)
        assert e.value.code == b.APB_ERR_SHAPE
    with pytest.raises(TypeError):
        b.apb_moe_route(z.t(), 2)
    with pytest.raises(ValueError):
        b.apb_moe_route(z, 2, workspace=torch.zeros(1, dtype=torch.int32, device="cuda"))
    row = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        b.apb_moe_combine(z, row)                                     # 4 rows, not 8
    with pytest.raises(TypeError):
        b.apb_moe_combine(torch.zeros(8, 8, device="cuda"), row.long())
    with pytest.raises(ValueError):
        b.apb_moe_combine(torch.zeros(8, 8, device="cuda"), row, torch.ones(4, device="cuda"))


@pytest.mark.parametrize("T,E,k", [(1, 9, 3), (40, 24, 4), (70, 300, 8)])
def test_route_gradient_by_differences_of_its_own_weights(b, T, E, k):
    """Central differences of apb_moe_route's weights, s = 1/8 and 1/16 combined so that their s^2 terms cancel.  In one logit a weight
    is a logistic function, the others what it leaves, and the fifth derivative of that function is 1/4 at most: s^4 / 480 * 1/4 * 2 max|d|
    is left.  Weights are within 64 * 2^-24 of themselves, so a difference is within 64 * 2^-24 / s and the two combined within three
    times that, of the sum of |d|; the gradient itself is within 128 * 2^-24 of twice that sum.  The logits lie 1/4 apart: no step
    changes their order, and all of them are exact."""
    g, s = np.random.default_rng(T + E), 2.0 ** -3
    z = torch.from_numpy(np.stack([g.permutation(E) for _ in range(T)]).astype(np.float32) / 4).cuda()
    d = torch.from_numpy(g.standard_normal((T, k)).astype(np.float32)).cuda()
    r = b.apb_moe_route(z, k)
    grad = b.apb_moe_route_backward(r["expert"], r["weight"], d, E).double()

    def loss(j, step):
        moved = z.scatter_add(1, r["expert"][:, j:j + 1].long(), torch.full((T, 1), step, device="cuda"))
        at = b.apb_moe_route(moved, k)
        assert torch.equal(at["expert"], r["expert"])
        return (at["weight"].double() * d.double()).sum(1)

    size = d.double().abs()
    tol = (3 * 64 / s + 256) * U * size.sum(1) + s ** 4 / 480 / 4 * 2 * size.amax(1)
    for j in range(k):
        diff = [(loss(j, h) - loss(j, -h)) / (2 * h) for h in (s, s / 2)]
        want = (4 * diff[1] - diff[0]) / 3
        got = grad.gather(1, r["expert"][:, j:j + 1].long())[:, 0]
        assert ((got - want).abs() <= tol).all()
    assert tol.max() < 0.01 * grad.abs().max()                       # (the tolerance says something)
