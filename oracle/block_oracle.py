"""Gated feed-forward blocks, 8-bit activation checkpoints and low-rank adapters in float64 (numpy), from their definitions."""
import numpy as np

ROOT = np.sqrt(2.0 / np.pi)


# ---- 8-bit blocks: values of a block of 32 are whole numbers times 2^e ------------------------------------------------

def quantize8(x):
    """x [rows, K] float32 -> (codes int8 [rows, Kp], scales uint8 [rows, Kp/32])."""
    x = np.asarray(x, dtype=np.float32)
    rows, K = x.shape
    v = np.zeros((rows, (K + 31) // 32 * 32), np.float64)
    v[:, :K] = x
    v = v.reshape(rows, -1, 32)
    top = np.abs(v).max(2)
    finite = np.isfinite(top)
    _, ex = np.frexp(np.where(finite & (top > 0), top, 1.0))
    e = np.where(top > 0, np.clip(ex - 1 - 6, -127, 121), -127)
    with np.errstate(invalid="ignore"):
        i = np.clip(np.rint(np.where(finite[..., None], v, 0.0) * np.exp2(-e.astype(np.float64))[..., None]), -127, 127)
    codes = np.where(finite[..., None], i, 0).astype(np.int8).reshape(rows, -1)
    return codes, np.where(finite, e + 127, 255).astype(np.uint8)


def values8(codes, scales, K):
    rows = codes.shape[0]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (codes.reshape(rows, -1, 32) * s[..., None]).reshape(rows, -1)[:, :K]


def pack8(codes, scales):
    return np.concatenate([codes.view(np.uint8).reshape(-1), scales.reshape(-1)])


def unpack8(mem, rows, K):
    blocks = (K + 31) // 32
    codes = mem[:rows * blocks * 32].view(np.int8).reshape(rows, blocks * 32)
    return codes, mem[rows * blocks * 32:rows * blocks * 33].reshape(rows, blocks)


# ---- activations --------------------------------------------------------------------------------------------------

def act(x, kind):
    """(act(x), act'(x), |z|, z'): z the argument of the sigmoid."""
    x = np.asarray(x, dtype=np.float64)
    if kind == "relu":
        return np.where(x < 0, 0.0, x), np.where(np.isnan(x), x, x > 0), np.zeros_like(x), np.zeros_like(x)
    with np.errstate(over="ignore", invalid="ignore"):
        z, dz = (x, np.ones_like(x)) if kind == "silu" else (2 * ROOT * (x + 0.044715 * x ** 3), 2 * ROOT * (1 + 0.134145 * x * x))
        small = np.exp(-np.abs(z))
        s = np.where(z >= 0, 1.0 / (1.0 + small), small / (1.0 + small))
        rest = np.where(z >= 0, small / (1.0 + small), 1.0 / (1.0 + small))      # 1 - s
        value = np.where(s == 0, 0.0, x * s)
        slope = s + np.where(s * rest == 0, 0.0, x * s * rest * dz)
    return value, slope, np.abs(z), dz


# ---- adapters --------------------------------------------------------------------------------------------------------

def rows_by_adapter(offsets, adapter, M, L):
    """The adapter of every row, -1 for none."""
    which = np.full(M, -1)
    offsets = [0, M] if offsets is None else offsets
    for s in range(len(offsets) - 1):
        a = s if adapter is None else int(adapter[s])
        which[offsets[s]:offsets[s + 1]] = a if 0 <= a < L else -1
    return which


def down(x, A, which, scale=None):
    """T, and the same with magnitudes."""
    M, r = x.shape[0], A.shape[1]
    T, mag = np.zeros((M, r)), np.zeros((M, r))
    for a in set(which[which >= 0].tolist()):
        rows = which == a
        s = 1.0 if scale is None else float(scale[a])
        T[rows] = s * (x[rows] @ A[a].T)
        mag[rows] = abs(s) * (np.abs(x[rows]) @ np.abs(A[a]).T)
    return T, mag


def up(T, B, which):
    out = np.zeros((T.shape[0], B.shape[2]))
    for a in set(which[which >= 0].tolist()):
        rows = which == a
        out[rows] = T[rows] @ B[a]
    return out


def gradient(T, x, which, L):
    out = np.zeros((L, T.shape[1], x.shape[1]))
    for a in set(which[which >= 0].tolist()):
        rows = which == a
        out[a] = T[rows].T @ x[rows]
    return out
