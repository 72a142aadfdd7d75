"""Microscaled 4-bit products, their gradients and the routing of tokens to experts, as cases that can be timed and compared.

A case is a dict of plain values: an operator, its sizes and its types.  `prepare` makes what a program holds before the
call, `run` makes one pass through the operator and returns everything it produced: with `own` set through the library's
entry points, without it in elementary torch operations in 32 bits, rounded once at the end.  `exact` is the same from the
definition in 64 bits.

Operators
  quantize   X -> blocks of 32 values with one power-of-two scale, each value in 4 bits; and back to the values they stand for
  linear     Y = Q(X) Q(W)^T, the activations quantized within the call
  grouped    the same for experts: row i of the product belongs to one expert and reads row row_token[i] of X
  backward   the gradients dX = G Q(W) and dW = G^T Q(X) at the quantized operands, plain or grouped by expert
  route      the k largest of E logits, softmax over them, rows grouped by expert; and the gradient of the logits
  combine    Y[t] = sum_j weight[t, j] Z[slot_row[t, j]]; and the gradients of Z and of the weights
"""
import math

import torch

own = False

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # activations of an odd batch in the library's K x M order (the 1000x517 classifier at batch 333): latency, and
        # blocks that lie across the contiguous axis
        dict(name="quantize 333x517 columns", op="quantize", M=333, K=517, type="f32", order="km"),
        # the activations of 16384 tokens, 4096 wide: a stream
        dict(name="quantize 16384x4096", op="quantize", M=16384, K=4096, type="bf16", order="mk"),
        # one new token through a 4096 x 4096 layer: the weights are all there is to read
        dict(name="linear one token 4096x4096", op="linear", M=1, N=4096, K=4096, type="bf16", out="bf16"),
        # a long prompt or a training batch through a wide layer: the matrix cores' work
        dict(name="linear 8192x8192x8192", op="linear", M=8192, N=8192, K=8192, type="bf16", out="bf16"),
        # a serving step: 16 sequences, 4 of 64 experts each, so most experts see one row or none
        dict(name="grouped 16 tokens 64 experts", op="grouped", T=16, E=64, k=4, N=2048, K=2048, skew=0.0, type="bf16", out="bf16"),
        # a long prompt: 8192 tokens to 2 of 16 experts, popular experts and odd sizes
        dict(name="grouped 8192 tokens 16 experts", op="grouped", T=8192, E=16, k=2, N=4099, K=4096, skew=1.0, type="bf16", out="bf16"),
        # training the odd classifier layer in 32 bits
        dict(name="backward 333x1000x517", op="backward", T=333, E=0, k=1, N=1000, K=517, skew=0.0, type="f32", out="f32"),
        # training the experts on 4096 tokens, 2 of 16 each
        dict(name="backward 4096 tokens 16 experts", op="backward", T=4096, E=16, k=2, N=4096, K=2048, skew=1.0, type="bf16", out="bf16"),
        # one new token's choice of experts: launches are all it costs
        dict(name="route one token", op="route", T=1, E=64, k=4, type="f32", masked=0.0),
        # a training batch's choice, with padding tokens that choose nothing
        dict(name="route 16384 tokens 128 experts", op="route", T=16384, E=128, k=8, type="bf16", masked=0.05),
        # one new token's experts joined
        dict(name="combine one token", op="combine", T=1, k=4, N=4096, type="bf16"),
        # a training batch's experts joined, and the gradients
        dict(name="combine 8192 tokens", op="combine", T=8192, k=4, N=4096, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "grouped", "grouped", "backward", "backward", "route", "combine"])
    types = ["f32", "bf16", "bf16", "f16"]
    while True:
        t, T, N, K = rng.choice(types), _log(rng, 1, 16384), _log(rng, 32, 8192), _log(rng, 32, 8192)
        E = _log(rng, 4, 128)
        k = rng.randint(1, min(8, E))
        if op == "quantize":
            if T * K <= 16384 * 4096:
                return dict(op=op, M=T, K=K, type=t, order=rng.choice(["mk", "mk", "km"]))
        elif op == "linear":
            if T <= 8192:
                return dict(op=op, M=T, N=N, K=K, type=t, out=rng.choice([t, "f32"]))
        elif op == "route":
            return dict(op=op, T=T, E=_log(rng, 4, 256), k=min(k, 8), type=t, masked=rng.choice([0.0, 0.05]))
        elif op == "combine":
            if T * k * N <= 8192 * 4 * 4096:
                return dict(op=op, T=T, k=k, N=N, type=t)
        else:
            if op == "backward" and rng.random() < 0.4:
                E, k = 0, 1
            most = 2 ** 38 if op == "grouped" else 2 ** 36
            if T * k * N * K <= most and max(E, 1) * N * K <= 2 ** 28 and T * k * (N + K) <= 2 ** 28:
                return dict(op=op, T=T, E=E, k=k, N=N, K=K, skew=rng.choice([0.0, 1.0]), type=t,
                            out=rng.choice([t, "f32"]))


# ---------------------------------------------------------------------------------------------------- inputs

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _acts(g, M, K):
    """Activations: normal, with channels of different spread and a few much larger ones."""
    spread = torch.exp(0.5 * _randn(g, K))
    spread = torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, spread * 10.0, spread)
    return _randn(g, M, K) * spread


def _groups(case, g):
    """Tokens' choices by popularity -> (row_token [R], offsets [E + 1], bounds: the offsets as a list)."""
    T, E, k = case["T"], case["E"], case["k"]
    popular = -case["skew"] * torch.log(torch.arange(1, E + 1, device="cuda").float())
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    expert = torch.topk(popular + noise, k, dim=1).indices
    order = torch.sort(expert.reshape(-1), stable=True).indices
    count = torch.bincount(expert.reshape(-1), minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(count, 0).int()
    return (order // k).int(), offsets, offsets.tolist()


def _inputs(case, seed):
    g, op = torch.Generator(device="cuda").manual_seed(seed), case["op"]
    dt = TYPE[case["type"]]
    s = dict(case)
    if op == "quantize":
        x = _acts(g, case["M"], case["K"]).to(dt)
        s["x"] = x.t().contiguous().t() if case["order"] == "km" else x
    elif op == "linear":
        s["x"] = _acts(g, case["M"], case["K"]).to(dt)
        s["w"] = _randn(g, case["N"], case["K"]) * 0.02
    elif op in ("grouped", "backward"):
        E = case["E"]
        s["row_token"], s["offsets"], s["bounds"] = _groups(case, g) if E else (None, None, [0, case["T"]])
        s["x"] = _acts(g, case["T"], case["K"]).to(dt)
        s["w"] = _randn(g, max(E, 1) * case["N"], case["K"]) * 0.02
        if op == "backward":
            s["g"] = (_randn(g, case["T"] * case["k"], case["N"]) * 1e-2).to(dt)
    elif op == "route":
        T, E = case["T"], case["E"]
        logits = _randn(g, T, E) * 2.0
        drop = torch.rand(T, E, generator=g, device="cuda") < case["masked"]     # experts out of reach of a token ...
        drop |= torch.rand(T, 1, generator=g, device="cuda") < case["masked"]    # ... and padding tokens
        s["logits"] = logits.masked_fill(drop, -math.inf).to(dt)
        s["dweight"] = _randn(g, T, case["k"])
    else:
        T, k, N = case["T"], case["k"], case["N"]
        s["z"], s["dy"] = _randn(g, T * k, N).to(dt), (_randn(g, T, N) * 1e-2).to(dt)
        s["slot_row"] = torch.randperm(T * k, generator=g, device="cuda").int().view(T, k)
        s["weight"] = torch.softmax(_randn(g, T, k), 1)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("linear", "grouped", "backward"):
        # the weights as a program keeps them; for the gradients also the activations as the forward pass left them
        w = s.pop("w")
        x = None
        if op == "backward":
            x = s.pop("x")
            x = x if s["row_token"] is None else x[s["row_token"].long()]
        if own:
            from paper_2306_08960_amd import binding as apb
            s["w4"] = apb.apb_mx4_quantize(w)
            if op == "backward":
                s["x4"] = apb.apb_mx4_quantize(x.contiguous())
            else:
                R = s["x"].shape[0] if op == "linear" else s["row_token"].numel()
                s["scratch"] = apb.alloc_mx4(R, case["K"])
        else:
            s["wq"] = _quantized(w)
            if op == "backward":
                s["xq"] = _quantized(x)
    elif op == "quantize" and own:
        from paper_2306_08960_amd import binding as apb
        s["mx"] = apb.alloc_mx4(case["M"], case["K"])
    elif op == "route" and own:
        from paper_2306_08960_amd import binding as apb
        s["workspace"] = apb.alloc_moe_workspace(case["T"], case["E"], case["k"])
    return s


# ---------------------------------------------------------------------------------------------------- plain forms

def _quantized(x):
    """The values that the 4-bit blocks of x stand for, in 32 bits."""
    M, K = x.shape
    pad = (-K) % 32
    v = torch.nn.functional.pad(x.float(), (0, pad)).view(M, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    e = (torch.frexp(top).exponent - 3).clamp(-120, 125)             # floor(log2(top)) - 2
    scale = torch.exp2(e.float())
    y = v.abs() / scale
    grid = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    q = (torch.round(y / grid) * grid).clamp(max=6.0)
    return (torch.where(v < 0, -q, q) * scale).view(M, K + pad)[:, :K]


def _plain_route(s):
    T, E, k = s["T"], s["E"], s["k"]
    logits = s["logits"].float()
    val, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    val, idx = val[:, :k], idx[:, :k]
    there = val > -math.inf
    top = torch.where(there[:, :1], val[:, :1], torch.zeros_like(val[:, :1]))
    p = torch.where(there, torch.exp(val - top), torch.zeros_like(val))
    weight = p / p.sum(1, keepdim=True).clamp(min=1e-30)
    expert = torch.where(there, idx, torch.full_like(idx, -1))
    key = torch.where(there, idx, torch.full_like(idx, E)).reshape(-1)
    order = torch.sort(key, stable=True).indices
    offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=key.device))
    slot_row = torch.empty_like(order)
    slot_row[order] = torch.arange(T * k, device=key.device)
    inner = (weight * s["dweight"]).sum(1, keepdim=True)
    g = torch.where(there, weight * (s["dweight"] - inner), torch.zeros_like(weight))
    dlogits = torch.zeros_like(logits)
    dlogits.scatter_(1, idx, g)
    return dict(expert=expert.int(), weight=weight, offsets=offsets.int(), row_token=(order // k).int(),
                slot_row=slot_row.view(T, k).int(), dlogits=dlogits.to(s["logits"].dtype))


def _plain(s):
    op = s["op"]
    if op == "quantize":
        return _quantized(s["x"]).to(s["x"].dtype)
    if op == "linear":
        return (_quantized(s["x"]) @ s["wq"].t()).to(TYPE[s["out"]])
    if op == "route":
        return _plain_route(s)
    if op == "combine":
        w, row = s["weight"], s["slot_row"].long()
        z, dy = s["z"].float()[row], s["dy"].float()
        y = (z * w[:, :, None]).sum(1)
        dz = torch.empty_like(s["z"])
        dz[row.view(-1)] = (dy[:, None, :] * w[:, :, None]).to(dz.dtype).view(-1, dz.shape[1])
        return dict(y=y.to(s["z"].dtype), dz=dz, dweight=(z * dy[:, None, :]).sum(2))
    N, out, bounds = s["N"], TYPE[s["out"]], s["bounds"]
    if op == "grouped":
        xq = _quantized(s["x"])[s["row_token"].long()]
        y = torch.empty(xq.shape[0], N, dtype=out, device="cuda")
        for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
            y[a:b] = (xq[a:b] @ s["wq"][e * N:(e + 1) * N].t()).to(out)
        return y
    g, xq, wq = s["g"].float(), s["xq"], s["wq"]
    dx, dw = torch.empty(xq.shape, dtype=out, device="cuda"), torch.empty_like(wq)
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        dx[a:b] = (g[a:b] @ wq[e * N:(e + 1) * N]).to(out)
        dw[e * N:(e + 1) * N] = g[a:b].t() @ xq[a:b]
    return dict(dx=dx, dw=dw)


# ---------------------------------------------------------------------------------------------------- the library's calls

def _own(s):
    from paper_2306_08960_amd import binding as apb
    op = s["op"]
    if op == "quantize":
        apb.apb_mx4_quantize(s["x"], mx=s["mx"])
        return apb.apb_mx4_dequantize(s["mx"], s["M"], s["K"], s["x"].dtype)
    if op == "linear":
        return apb.apb_mx4_linear(s["x"], s["w4"], s["N"], dtype=TYPE[s["out"]], scratch=s["scratch"])
    if op == "grouped":
        return apb.apb_mx4_linear(s["x"], s["w4"], s["N"], dtype=TYPE[s["out"]], scratch=s["scratch"],
                                  rows_from=s["row_token"], offsets=s["offsets"])
    if op == "backward":
        dx = apb.apb_mx4_backward_input(s["g"], s["w4"], s["K"], dtype=TYPE[s["out"]], offsets=s["offsets"])
        dw = apb.apb_mx4_backward_weight(s["g"], s["x4"], s["K"], offsets=s["offsets"])
        return dict(dx=dx, dw=dw)
    if op == "route":
        r = apb.apb_moe_route(s["logits"], s["k"], workspace=s["workspace"])
        r["dlogits"] = apb.apb_moe_route_backward(r["expert"], r["weight"], s["dweight"], s["E"], s["logits"].dtype)
        return r
    y = apb.apb_moe_combine(s["z"], s["slot_row"], s["weight"])
    dz, dweight = apb.apb_moe_combine_backward(s["dy"], s["z"], s["slot_row"], s["weight"])
    return dict(y=y, dz=dz, dweight=dweight)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------- work

def work(case):
    op = case["op"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    s = size[case["type"]]
    mx = 0.5 + 1.0 / 32                                              # bytes of a quantized value with its share of a scale
    if op == "quantize":                                             # x read, x^ written in its type; the 4-bit form both ways
        n = case["M"] * case["K"]
        return {"bytes": n * (2 * s + 2 * mx), "flops": 4.0 * n}
    if op == "route":                                                # logits and dweight read; dlogits and six small arrays written
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": 2.0 * s * T * E + 4.0 * T * k * 5 + 4.0 * (E + 1), "flops": 2.0 * T * E}
    if op == "combine":                                              # z and dy read, y and dz written
        T, k, N = case["T"], case["k"], case["N"]
        return {"bytes": s * 2.0 * N * (T * k + T) + 4.0 * T * k * 3, "flops": 5.0 * T * k * N}
    N, K, o = case["N"], case["K"], size[case["out"]]
    if op == "linear":
        M = case["M"]
        return {"bytes": s * M * K + mx * N * K + o * M * N, "flops": 2.0 * M * N * K}
    R, E = case["T"] * case["k"], max(case["E"], 1)
    if op == "grouped":
        reached = E * (1.0 - (1.0 - case["k"] / E) ** case["T"])     # experts that have a row, were all alike
        return {"bytes": s * case["T"] * K + mx * reached * N * K + o * R * N + 8.0 * R, "flops": 2.0 * R * N * K}
    return {"bytes": s * 2.0 * R * N + mx * (R * K + E * N * K) + o * R * K + 4.0 * E * N * K, "flops": 4.0 * R * N * K}


# ---------------------------------------------------------------------------------------------------- 64 bits

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_quantized(x):
    """Definition in 64 bits: the largest power of two not above the block's largest magnitude, divided by 4, is the scale;
    every value goes to the nearest level, a value midway to the level of even index."""
    M, K = x.shape
    v = torch.zeros(M, (K + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    v[:, :K] = x
    v = v.view(M, -1, 32)
    mantissa, exponent = torch.frexp(v.abs().max(2).values)
    scale = torch.ldexp(torch.full_like(mantissa, 0.125), exponent).unsqueeze(2)
    y = v.abs() / scale
    index = torch.zeros_like(y, dtype=torch.int32)
    for i in range(7):
        mid = (LEVELS[i] + LEVELS[i + 1]) / 2
        index += (y > mid) if i % 2 == 0 else (y >= mid)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[index.long()]
    return (torch.sign(v) * level * scale).view(M, -1)[:, :K]


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "quantize":
        return _exact_quantized(s["x"])
    if op == "linear":
        return torch.mm(_exact_quantized(s["x"]), _exact_quantized(s["w"]).t().contiguous())
    if op == "route":
        return _exact_route(s)
    if op == "combine":
        w, row, dy = s["weight"].double(), s["slot_row"].long(), s["dy"].double()
        y, dz, dw = torch.zeros_like(dy), torch.zeros_like(s["z"], dtype=torch.float64), torch.zeros_like(w)
        for j in range(case["k"]):
            z = s["z"].double()[row[:, j]]
            y += w[:, j:j + 1] * z
            dz[row[:, j]] = w[:, j:j + 1] * dy
            dw[:, j] = torch.linalg.vecdot(z, dy)
        return dict(y=y, dz=dz, dweight=dw)
    N, K, R, ends = case["N"], case["K"], case["T"] * case["k"], s["bounds"]
    token = torch.arange(R, device="cuda") if s["row_token"] is None else s["row_token"].long()
    xq = _exact_quantized(s["x"])
    if op == "grouped":
        y = torch.zeros(R, N, dtype=torch.float64, device="cuda")
    else:
        dx = torch.zeros(R, K, dtype=torch.float64, device="cuda")
        dw = torch.zeros(max(case["E"], 1) * N, K, dtype=torch.float64, device="cuda")
    for e in range(len(ends) - 1):
        rows, at = slice(ends[e], ends[e + 1]), slice(e * N, (e + 1) * N)
        w = _exact_quantized(s["w"][at])
        if op == "grouped":
            y[rows] = torch.mm(xq[token[rows]], w.t().contiguous())
        else:
            g = s["g"][rows].double()
            dx[rows] = torch.mm(g, w)
            dw[at] = torch.mm(g.t().contiguous(), xq[token[rows]])
    return y if op == "grouped" else dict(dx=dx, dw=dw)


def _exact_route(s):
    """One choice after another: the largest logit not yet taken, the lowest index among equals."""
    T, E, k = s["T"], s["E"], s["k"]
    left = s["logits"].double().clone()
    each = torch.arange(E, device="cuda").expand(T, E)
    expert, value = [], []
    for _ in range(k):
        top = left.amax(1, keepdim=True)
        first = torch.where(left == top, each, E).amin(1, keepdim=True)
        value.append(top)
        expert.append(torch.where(top == -math.inf, -1, first))
        left.scatter_(1, first, -math.inf)
    expert, value = torch.cat(expert, 1), torch.cat(value, 1)
    weight = torch.nan_to_num(torch.softmax(value, 1), nan=0.0)
    dlogits = torch.zeros(T, E + 1, dtype=torch.float64, device="cuda")
    dw = s["dweight"].double()
    dlogits.scatter_add_(1, torch.where(expert < 0, E, expert), weight * dw - weight * (weight * dw).sum(1, keepdim=True))
    flat = torch.where(expert < 0, E, expert).reshape(-1)
    row = torch.argsort(flat * (T * k) + torch.arange(T * k, device="cuda"))
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cumsum(torch.bincount(flat, minlength=E + 1), 0)])
    slot_row = torch.zeros(T * k, dtype=torch.int64, device="cuda").scatter_(0, row, torch.arange(T * k, device="cuda"))
    return dict(expert=expert.int(), weight=weight, offsets=offsets[:E + 1].int(),
                row_token=torch.div(row, k, rounding_mode="floor").int(), slot_row=slot_row.view(T, k).int(),
                dlogits=dlogits[:, :E])
