"""Sizes by which the products of 4-bit matrices reach every tile size, and the offsets of their groups.  The host
test checks that the rules send them there, the GPU tests what comes out."""
import numpy as np

# M, N, K, E (0: no groups), side of the product's tiles.  Ragged in every direction; a K of one segment is fewer passes than the
# product keeps under way.
PRODUCTS = [
    (130, 300, 520, 0, 64),
    (1700, 2050, 300, 0, 128), (1540, 1801, 40, 0, 128), (1700, 2050, 1300, 5, 128),
    (3400, 3601, 520, 0, 256), (3330, 3650, 33, 0, 256), (3400, 3601, 777, 4, 256),
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
