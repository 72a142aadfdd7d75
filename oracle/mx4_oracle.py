"""CPU oracle for the microscaled 4-bit matrices and the routing of tokens to experts -- TEST INFRASTRUCTURE ONLY.

Plain numpy in float64, written from the definitions; nothing here is shared with, or imported by, the HIP library.

  quantize        block of 32 along the last axis: e = clamp(floor(log2 max|x|) - 2, -127, 125); level = the nearest of LEVELS to
                  |x| / 2^e, midway to the even index, 6 beyond; a block with a non-finite value has scale code 255
  values          (-1)^sign * level * 2^e, NaN for scale code 255
  product         Y[m] = W^[e] X^[m] with the expert e of row m; rows that belong to none: 0
  gradients       dX[m] = G[m] W^[e];  dW[e] = sum over the rows of e of G[m] (outer) X^[m]
  route           k largest logits, ties to the lowest index, -inf and NaN never; softmax over them; stable order by expert
  combine         Y[t] = sum_j w[t, j] Z[slot_row[t, j]]
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK, SEG = 32, 256


def quantize(x: np.ndarray):
    """x [rows, K] float32 -> (codes uint8 [rows, Kp] with bit 3 the sign, scales uint8 [rows, Kp / 32]); Kp = K in whole
    segments of 256."""
    x = np.asarray(x, dtype=np.float32)
    rows, K = x.shape
    Kp = (K + SEG - 1) // SEG * SEG
    v = np.zeros((rows, Kp), dtype=np.float64)
    v[:, :K] = x
    v = v.reshape(rows, Kp // BLOCK, BLOCK)
    top = np.max(np.abs(v), axis=2)
    bad = ~np.isfinite(v).all(axis=2)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.frexp(safe)[1] - 1 - 2                                  # frexp: top = f * 2^n with f in [1/2, 1)
    e = np.where(top == 0, -127, np.clip(e, -127, 125))
    y = np.abs(np.where(bad[:, :, None], 0.0, v)) / np.ldexp(1.0, e)[:, :, None]
    below = np.clip(np.searchsorted(LEVELS, y, side="right") - 1, 0, 6)
    lo, hi = LEVELS[below], LEVELS[below + 1]
    up = (y - lo > hi - y) | ((y - lo == hi - y) & (below % 2 == 1))
    level = below + up
    codes = np.where(bad[:, :, None], 0, level + 8 * np.signbit(v)).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return codes.reshape(rows, Kp), scales


def values(codes: np.ndarray, scales: np.ndarray, K: int) -> np.ndarray:
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0) * np.repeat(scale, BLOCK, axis=1)
    return v[:, :K]


def quantized(x: np.ndarray) -> np.ndarray:
    """The values that the 4-bit form of x stands for, float64."""
    return values(*quantize(x), np.asarray(x).shape[1])


def pack(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The bytes of a 4-bit matrix in memory: two codes to a byte, even column low; then scales by segment, row, block."""
    rows, Kp = codes.shape
    pairs = codes.reshape(rows, Kp // 2, 2)
    body = (pairs[:, :, 0] | pairs[:, :, 1] << 4).astype(np.uint8)
    tail = scales.reshape(rows, Kp // SEG, 8).transpose(1, 0, 2)
    return np.concatenate([body.reshape(-1), np.ascontiguousarray(tail).reshape(-1)])


def _bounds(offsets, M):
    return [0, M] if offsets is None else [int(o) for o in offsets]


def product(xq: np.ndarray, wq: np.ndarray, N: int, offsets=None):
    """(Y, sum of the magnitudes of Y's terms); xq [M, K], wq [E * N, K]."""
    M = xq.shape[0]
    y, mag = np.zeros((M, N)), np.zeros((M, N))
    b = _bounds(offsets, M)
    for e in range(len(b) - 1):
        w = wq[e * N:(e + 1) * N]
        y[b[e]:b[e + 1]] = xq[b[e]:b[e + 1]] @ w.T
        mag[b[e]:b[e + 1]] = np.abs(xq[b[e]:b[e + 1]]) @ np.abs(w).T
    return y, mag


def gradients(g: np.ndarray, xq: np.ndarray, wq: np.ndarray, offsets=None):
    """(dX, dW, magnitudes of dX's terms, of dW's)."""
    g = np.asarray(g, dtype=np.float64)
    M, N = g.shape
    dx, dw, mx, mw = np.zeros(xq.shape), np.zeros(wq.shape), np.zeros(xq.shape), np.zeros(wq.shape)
    b = _bounds(offsets, M)
    for e in range(len(b) - 1):
        r, n = slice(b[e], b[e + 1]), slice(e * N, (e + 1) * N)
        dx[r], mx[r] = g[r] @ wq[n], np.abs(g[r]) @ np.abs(wq[n])
        dw[n], mw[n] = g[r].T @ xq[r], np.abs(g[r]).T @ np.abs(xq[r])
    return dx, dw, mx, mw


def route(logits: np.ndarray, k: int) -> dict:
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    expert, weight = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    for t in range(T):
        can = [e for e in range(E) if logits[t, e] > -np.inf]        # False for NaN
        chosen = sorted(can, key=lambda e: (-logits[t, e], e))[:k]
        if chosen:
            p = np.exp(logits[t, chosen] - logits[t, chosen[0]])
            expert[t, :len(chosen)], weight[t, :len(chosen)] = chosen, p / p.sum()
    flat = np.where(expert < 0, E, expert).reshape(-1)
    order = np.argsort(flat, kind="stable")
    slot_row = np.empty(T * k, dtype=np.int64)
    slot_row[order] = np.arange(T * k)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E + 1))])[:E + 1]
    return {"expert": expert, "weight": weight, "offsets": offsets, "row_token": order // k, "slot_row": slot_row.reshape(T, k)}


def route_backward(expert: np.ndarray, weight: np.ndarray, dweight: np.ndarray, E: int) -> np.ndarray:
    T, k = expert.shape
    out = np.zeros((T, E))
    w, d = np.asarray(weight, dtype=np.float64), np.asarray(dweight, dtype=np.float64)
    for t in range(T):
        inner = sum(w[t, j] * d[t, j] for j in range(k) if expert[t, j] >= 0)
        for j in range(k):
            if expert[t, j] >= 0:
                out[t, expert[t, j]] = w[t, j] * (d[t, j] - inner)
    return out


def combine(z: np.ndarray, slot_row: np.ndarray, weight: np.ndarray) -> np.ndarray:
    z, y = np.asarray(z, dtype=np.float64), np.zeros((slot_row.shape[0], z.shape[1]))
    for j in range(slot_row.shape[1]):
        live = weight[:, j] != 0
        y[live] += np.asarray(weight, dtype=np.float64)[live, j:j + 1] * z[slot_row[live, j]]
    return y


def combine_backward(dy: np.ndarray, z: np.ndarray, slot_row: np.ndarray, weight: np.ndarray):
    dy, z = np.asarray(dy, dtype=np.float64), np.asarray(z, dtype=np.float64)
    dz, dw = np.zeros(z.shape), np.zeros(slot_row.shape)
    for j in range(slot_row.shape[1]):
        w = np.asarray(weight, dtype=np.float64)[:, j:j + 1]
        dz[slot_row[:, j]] = np.where(w == 0, 0.0, w * dy)
        dw[:, j] = (dy * z[slot_row[:, j]]).sum(1)
    return dz, dw
