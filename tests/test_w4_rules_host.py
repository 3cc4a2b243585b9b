"""Which kernels products by 4-bit weights take, on the host (the figures are times in us
on the GPU)."""
import pytest

from test_glu_host_runtime import driver, launched  # noqa: F401 (a fixture)

# n, d, f, precision, group, and the call; what the kernel for few rows and tiles take:
# they differ by a tenth or more.
FEW_ROWS = [
    (1, 4096, 8192, 2, 128, "w4"),       # 6.9, 60
    (1, 4096, 65536, 2, 128, "w4"),      # 30, 70
    (1, 4096, 131072, 2, 128, "w4"),     # 58, 150
    (8, 4096, 131072, 2, 128, "w4"),     # 63, 150
    (16, 8192, 65536, 2, 128, "w4"),     # 78, 150
    (1, 8192, 1024, 2, 128, "w4"),       # 5.9, 113
    (1, 4096, 32768, 2, 128, "w4_glu"),  # 31, 78
    (1, 4096, 131072, 2, 128, "w4_glu"), # 115, 290
    (1, 8192, 65536, 0, 32, "w4_glu"),   # 292, 441
    (1, 256, 8192, 2, 128, "w4"),        # 3.0, 8.6
    (32, 256, 8192, 2, 128, "w4"),       # 3.6, 9.3
    (16, 128, 8192, 2, 32, "w4"),        # 3.1, 7.6
    (1, 64, 4096, 2, 32, "w4"),          # 3.2, 8.6
    (64, 40, 700, 2, 128, "w4"),         # 3.4, 10
    (48, 40, 700, 0, 128, "w4"),         # 3.8, 8.7
    (64, 64, 4096, 2, 128, "w4"),        # 3.8, 9.8
]
TILES = [
    (16, 128, 131072, 0, 32, "w4_glu"),  # 73, 35
    (64, 256, 65536, 2, 128, "w4"),      # 25, 14
    (64, 4096, 32768, 2, 32, "w4_glu"),  # 190, 124
    (512, 4096, 8192, 2, 128, "w4"),     # 131, 66
    (512, 1024, 32768, 1, 32, "w4_glu"), # 535, 136
    (1000, 301, 20000, 2, 128, "w4"),    # 196, 58: rows of an odd length
]


@pytest.mark.parametrize("case", FEW_ROWS, ids=str)
def test_few_rows(driver, case):  # noqa: F811
    line, = launched(driver, [(case[5], *case[:5])])
    assert "rows_kernel" in line and "w4_tile" not in line, line


@pytest.mark.parametrize("case", TILES, ids=str)
def test_tiles(driver, case):  # noqa: F811
    line, = launched(driver, [(case[5], *case[:5])])
    assert "w4_tile" in line, line


def test_sizes_of_the_range_tests(driver):  # noqa: F811
    """test_w4_range_gpu.py is about tiles too: its largest sizes take them, in each type
    and group that it has."""
    calls = [(op, 2900, 700, 1500, p, g) for op in ("w4", "w4_glu") for p in (0, 2) for g in (32, 64, 128)]
    calls += [("w4", 6000, 40, 700, p, 32) for p in (0, 1, 2)]
    assert all("w4_tile" in line for line in launched(driver, calls))


def test_blocks_by_groups_of_32(driver):  # noqa: F811
    """Two tiles and 16 rows of fp32 spill registers: 133 us, one tile 83."""
    one, = launched(driver, [("w4_glu", 1, 4096, 32768, 0, 32)])
    two, = launched(driver, [("w4_glu", 1, 4096, 32768, 0, 64)])
    assert "rows_kernelIfLi32ELb1ELi1ELi1E" in one and "rows_kernelIfLi64ELb1ELi2ELi1E" in two, (one, two)
