"""Sizes by which the products of 4-bit matrices and their gradients reach every tile size, and the offsets of their groups.  The
host test checks that the rules send them there, the GPU tests what comes out."""
import numpy as np

# M, N, K, E (0: no groups), side of the product's tiles.  Ragged in every direction; a K of one segment is fewer passes than the
# product keeps under way.
PRODUCTS = [
    (130, 300, 520, 0, 64),
    (1700, 2050, 300, 0, 128), (1540, 1801, 40, 0, 128), (1700, 2050, 1300, 5, 128),
    (3400, 3601, 520, 0, 256), (3330, 3650, 33, 0, 256), (3400, 3601, 777, 4, 256),
]

# M, N, K, E, type of the gradient, then for dX and dW: tiles of 64 * f a side, groups of waves, slices.  Sums of odd and even numbers
# of passes of 64, the last one never whole; an N of whole blocks (1032, 2500) and others.
GRADIENTS = [
    (2000, 2050, 1900, 0, "bf16", (2, 2, 1), (2, 2, 1)), (2000, 2050, 1900, 0, "f32", (2, 1, 1), (2, 1, 1)),
    (2000, 2050, 1900, 0, "f16", (2, 1, 1), (2, 1, 1)),
    (2500, 2050, 2500, 0, "bf16", (2, 1, 1), (2, 1, 1)),
    (510, 4100, 4000, 0, "bf16", (2, 1, 2), (4, 1, 1)), (510, 4100, 4000, 0, "f32", (2, 1, 2), (2, 1, 1)),
    (510, 4100, 4000, 0, "f16", (2, 1, 2), (2, 1, 1)),
    (8200, 1030, 1000, 0, "bf16", (2, 1, 1), (2, 1, 3)), (8200, 1030, 1000, 0, "f32", (2, 1, 1), (2, 1, 3)),
    (8200, 1030, 1000, 0, "f16", (2, 1, 1), (2, 1, 3)),
    (4133, 2500, 2500, 0, "bf16", (4, 1, 1), (4, 1, 2)),
    (2500, 4133, 2500, 0, "bf16", (4, 1, 2), (4, 1, 1)),
    (3400, 1032, 2600, 4, "bf16", (4, 1, 1), (4, 1, 1)),
    (2000, 1026, 1900, 3, "bf16", (2, 2, 1), (2, 1, 1)), (2000, 1026, 1900, 3, "f32", (2, 1, 1), (2, 1, 1)),
    (500, 4100, 2000, 2, "bf16", (2, 1, 3), (4, 1, 1)), (500, 4100, 2000, 2, "f16", (2, 1, 4), (2, 1, 1)),
    (8200, 1030, 520, 2, "bf16", (2, 1, 1), (2, 1, 2)), (8200, 1030, 520, 2, "f32", (2, 1, 1), (2, 1, 2)),
]

# The same for a 4-bit matrix with blocks of NaN and of the smallest and largest scales: each tile size with whole passes of 64 and with
# sums shorter than that.
SPECIAL = [
    (40, 50, 300, "bf16", (1, 2, 1), (1, 2, 1)), (40, 50, 300, "f32", (1, 2, 1), (1, 2, 1)),
    (200, 300, 520, "bf16", (1, 2, 1), (1, 2, 1)), (200, 300, 520, "f16", (1, 2, 1), (1, 2, 1)), (200, 300, 520, "f32", (1, 2, 1), (1, 2, 1)),
    (2050, 40, 1900, "bf16", (2, 2, 1), (1, 2, 8)), (40, 2050, 1900, "f32", (1, 2, 8), (2, 1, 1)),
    (1700, 130, 1900, "bf16", (2, 2, 1), (1, 2, 2)), (1700, 130, 1900, "f16", (2, 1, 1), (1, 2, 2)), (1700, 130, 1900, "f32", (2, 1, 1), (1, 2, 2)),
    (130, 1700, 1900, "bf16", (1, 2, 2), (2, 2, 1)), (130, 1700, 1900, "f32", (1, 2, 2), (2, 1, 1)),
    (3400, 130, 2600, "bf16", (4, 1, 1), (1, 2, 2)), (130, 3400, 2600, "bf16", (1, 2, 2), (4, 1, 1)),
    (3400, 40, 2600, "bf16", (4, 1, 1), (1, 2, 6)), (40, 3400, 2600, "bf16", (1, 2, 6), (4, 1, 1)),
]


def offsets(M, E):
    """An expert of 3/5 of the rows, one without any, one of 30, the others alike; ten rows belong to none."""
    if E == 0:
        return None
    rows = [M * 3 // 5, 0, 30] + [0] * (E - 3) if E >= 3 else [M * 3 // 5] + [0] * (E - 1)
    left = M - 10 - sum(rows)
    alike = range(3, E) if E > 3 else [E - 1]
    for e in alike:
        rows[e] += left // len(alike)
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
