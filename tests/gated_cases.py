"""Sizes by which the gated products reach every tile size, plain and grouped, and the kernel for few rows and little work."""

# M, N, K, E (0: no groups), side of the tiles (which a call takes that saves both projections, or has much work).  Ragged in every
# direction.
PRODUCTS = [
    (1, 1, 1, 0, 64), (16, 130, 8193, 0, 64), (1, 17, 300, 0, 64), (16, 33, 256, 0, 64), (16, 4100, 4096, 0, 64),
    (7, 1000, 9000, 0, 64), (17, 15, 31, 0, 64), (130, 150, 520, 0, 64), (300, 700, 2600, 0, 64), (64, 32, 257, 0, 64),
    (200, 47, 1300, 3, 64), (1700, 1025, 300, 0, 128), (1540, 901, 40, 0, 128), (1700, 1025, 1300, 5, 128), (3400, 1801, 520, 0, 256),
    (3330, 1825, 33, 0, 256), (3400, 1801, 777, 4, 256),
]
