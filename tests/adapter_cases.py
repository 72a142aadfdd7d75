"""Sizes by which the adapters' kernels are reached in every form, and their segments.  The host test checks that the rules send them
there, the GPU tests what comes out."""
import numpy as np

# M, K, N, r, L, segments: every number of ranks and rows to a workgroup, parts of sums, slices; ragged in every direction, and whole
CASES = [
    (1, 1, 1, 1, 1, "all"), (1, 4096, 4096, 16, 3, "all"), (1, 1000, 517, 5, 2, "tokens"), (64, 4096, 600, 16, 8, "tokens"),
    (33, 517, 1000, 3, 2, "mixed"), (100, 300, 130, 17, 4, "mixed"), (40, 64, 512, 33, 5, "own"), (16, 70, 31, 64, 2, "mixed"),
    (333, 517, 1000, 16, 2, "mixed"), (900, 1000, 515, 8, 3, "own"), (700, 2048, 1100, 32, 1, "all"), (1500, 300, 260, 64, 3, "mixed"),
    (2600, 40, 24, 4, 1, "all"), (4096, 16, 40, 3, 7, "tokens"), (3000, 5, 6, 18, 2, "mixed"),
    (400, 200, 140, 100, 2, "mixed"), (300, 96, 520, 256, 2, "all"),
    (4100, 40, 8200, 12, 3, "mixed"), (2100, 40, 8200, 30, 3, "mixed"), (4200, 60, 8200, 50, 1, "all"), (4100, 128, 8192, 64, 2, "mixed"),
    (4100, 24, 8300, 100, 2, "mixed"), (2100, 24, 8300, 200, 2, "mixed"), (4100, 24, 8192, 20, 2, "own"),
    (12100, 40, 30, 9, 3, "mixed"), (9000, 70, 50, 30, 2, "mixed"), (9000, 70, 40, 100, 2, "mixed"), (700, 8300, 40, 20, 2, "mixed"),
    (40, 4100, 100, 70, 30, "own"), (2000, 130, 70, 20, 9, "many"), (8, 9000, 100, 130, 4, "tokens"),
    (600, 200, 40, 10, 7, "mixed"), (600, 130, 30, 24, 7, "own"), (500, 150, 50, 60, 9, "mixed"), (1300, 4100, 40, 12, 8, "own"),
    (1100, 8300, 48, 30, 4, "own"), (9000, 4100, 16, 9, 8, "same"), (50, 30, 20, 40, 3, "mixed"), (70, 24, 40, 20, 4, "own"),
    (300, 60, 9, 16, 2, "many"), (1747, 30, 40, 130, 3, "many"), (1422, 40, 30, 256, 3, "mixed"),
    (600, 4100, 70, 12, 24, "mixed"), (1500, 300, 40, 9, 220, "mixed"), (300, 517, 1000, 70, 70, "all"), (70, 2000, 24, 20, 150, "many"),
]


def segments(kind, M, L, seed):
    """(offsets, adapter): requests of one token, of any length with empty ones and rows behind the last, all rows, one per adapter,
    all of one adapter."""
    g = np.random.default_rng(seed)
    if kind == "all":
        return None, np.array([L - 1], np.int32)
    if kind == "tokens":
        return np.arange(M + 1, dtype=np.int32), g.integers(-1, L + 1, M).astype(np.int32)
    S = L if kind in ("own", "same") else 70 if kind == "many" else 6
    cut = np.sort(g.integers(0, M - M // 8 + 1, S))
    off = np.concatenate([[0], cut]).astype(np.int32)
    if S > 2:
        off[2] = off[1]
    if kind == "same":
        off[-1] = M
        return off, np.full(S, L - 1, np.int32)
    return off, None if kind == "own" else g.integers(-1, L, S).astype(np.int32)
