"""Sizes at which the gated block and products by 4-bit weights take each of their
kernels (test_glu_host_runtime.py checks that they do; the tests on the GPU run
them)."""

# The block and its gradient (n, d, f): single rows, few by 16, 32 and 64, tiles; nothing is a whole
# number of tiles or steps, rows of odd lengths and of whole 16 bytes, one
# coordinate, one result.
GLU = [(1, 1, 1), (1, 40, 300), (1, 301, 77), (2, 129, 33), (5, 1000, 16), (16, 128, 130), (17, 64, 257), (33, 7, 19),
       (64, 520, 100), (65, 520, 100), (100, 33, 129), (257, 301, 300), (300, 1, 5), (130, 256, 1), (1000, 100, 511),
       (60, 1001, 2041), (700, 130, 1300)]
# Enough tiles for the largest: of h, of dx, of dw.
LARGE = [(4100, 40, 2060), (4100, 2090, 130), (130, 1300, 2900)]

# Products by 4-bit weights (n, d, f).
W4 = [(1, 1, 1), (1, 40, 300), (1, 1301, 77), (3, 129, 33), (7, 2000, 15), (16, 128, 130), (17, 64, 257), (33, 7, 19),
      (64, 520, 100), (65, 384, 100), (200, 301, 70), (300, 1000, 530)]
# Enough rows for tiles through LDS: several blocks of 128 coordinates and one of less,
# one block, one coordinate.
W4_LARGE = [(2900, 700, 1500), (2500, 520, 150), (3000, 100, 700), (6000, 1, 40)]
# Rows (n, d) whose values in each type fill half the last-level cache.
W4_BACK = (16_500, 4101)
