"""Sizes at which the calls on microscaled rows take each of their kernels
(test_mx_host_runtime.py checks that they do; the tests on the GPU run them)."""

# Products (m, n, d): few results, then tiles of 64 x 128, 128 x 128, 128 x 256 and,
# with A of 4 bits, 256 x 256; nothing is a whole number of tiles or steps.
PRODUCTS = [(1, 333, 700), (19, 1001, 260), (130, 8191, 500), (300, 9000, 700), (1031, 12_001, 400), (1030, 12_101, 1500)]

# Sets (n, d, l, k).  Rows of every number of 128 coordinates that has kernels of
# its own, and of one less where two share them.  Of each: many points, several set
# groups to a workgroup, an odd number of members, the last group not full; few
# points and groups; one block of points and very many groups.
SETS_D = [100, 250, 383, 500, 620, 700, 800, 1000, 1100, 1250, 1400, 1500, 1650, 1700, 1900, 2000]
SETS = [(n, d, l, k) for d in SETS_D for n, l, k in ((40_011, 300, 7), (3001, 100, 19), (100, 30_001, 3))]
# Rows short enough for workgroups that stage their sets themselves, and too long
# for all the others.
SETS += [(10_000, 60, 45, 8), (4001, 200, 45, 5), (3001, 2176, 100, 5), (130, 4100, 300, 9)]

# Gradients of the norm (n, d), each kernel with so many rows that a thread takes
# several of them after each other: 512 workgroups of 16, 4 or 1 rows at a time.
GRADIENTS = [(17_003, 100), (8300, 256), (2100, 500), (4150, 1000), (2500, 1303), (2051, 2048), (1300, 2049), (1037, 4096),
             (1025, 5003), (530, 8192), (70, 8200)]

# Rounding there and back (n, d): results that fit the last-level cache, and more
# than 256 MiB of them in every type.
ROUNDINGS = [(65, 100), (300_007, 499)]
