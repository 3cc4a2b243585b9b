"""Sizes at which the calls on microscaled rows take each of their kernels
(test_mx_host_runtime.py checks that they do; the tests on the GPU run them)."""

# Products (m, n, d): few results, then tiles of 64 x 128, 128 x 128, 128 x 256 and,
# with A of 4 bits, 256 x 256; nothing is a whole number of tiles or steps.
PRODUCTS = [(1, 333, 700), (19, 1001, 260), (130, 8191, 500), (300, 9000, 700), (1031, 12_001, 400), (1030, 12_101, 1500)]
