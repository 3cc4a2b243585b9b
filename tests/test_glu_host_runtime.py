"""The host code of the gated block and of the calls on 4-bit weights over a HIP
runtime that launches nothing (tests/fake_hip/glu_driver.cpp), without a GPU."""
import os
import re
import subprocess

import pytest

import glu_sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = ("dense_", "rows_kernel", "w4_", "glu_point", "zero_bytes")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    from paper_2101_08763_amd import build as B
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not available")
    os.makedirs(B.OBJDIR, exist_ok=True)
    objs = []
    for src in B.SOURCES:
        obj = os.path.join(B.OBJDIR, os.path.splitext(src)[0] + ".o")
        if not os.path.exists(obj):
            B._compile(src, False)
        objs.append(obj)
    tmp = tmp_path_factory.mktemp("fake_hip_glu")
    drv, exe = str(tmp / "driver.o"), str(tmp / "driver")
    for cmd in ([B.HIPCC, "-O1", "-std=c++17", f"-I{B.INCLUDE}", "-Wno-unused-value", "-Wno-unused-function", "-c",
                 os.path.join(ROOT, "tests", "fake_hip", "glu_driver.cpp"), "-o", drv],
                [B.HIPCC, f"--offload-arch={B.ARCH}", drv, *objs, "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stdout + r.stderr
    return exe


def run(driver, *args, stdin=""):
    env = {k: v for k, v in os.environ.items() if not k.startswith("EXEMCL_")}
    return subprocess.run([driver, *args], input=stdin, capture_output=True, text=True, timeout=300, env=env)


@pytest.mark.parametrize("check", ["capture", "grids", "limits"])
def test_host_runtime(driver, check):
    r = run(driver, check)
    assert r.returncode == 0 and "checks passed" in r.stdout, r.stdout + r.stderr


def names(text):
    """The kernels of this part of the library among symbols."""
    return {s.split(":")[0] for s in text.split() if re.search(r"\d(dense_\w+?_kernel|dense_kernel|rows_kernel|w4_\w+?_kernel|"
                                                               r"glu_point_kernel|zero_bytes_kernel)", s)}


def launched(driver, calls):
    r = run(driver, "calls", stdin="".join(" ".join(map(str, c)) + "\n" for c in calls))
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout.splitlines()[:-1]


def test_sizes_of_the_tests_take_every_kernel(driver):
    """A kernel that is compiled is run by the tests on the GPU, whatever the rule that
    chooses it."""
    precs, groups = (0, 1, 2), (32, 64, 128)
    calls = [("glu", *s, p, 0) for s in glu_sizes.GLU + glu_sizes.LARGE for p in precs]
    calls += [("grad", *s, p, i % 4) for i, s in enumerate(glu_sizes.GLU) for p in precs]
    calls += [("grad", *s, p, 0) for s in glu_sizes.LARGE for p in precs]
    calls += [(op, *s, p, g) for op in ("w4", "w4_glu") for s in glu_sizes.W4 + glu_sizes.W4_LARGE for p in precs for g in groups]
    calls += [(op, 70, 1000, 0, p, g) for op in ("quantize", "dequantize") for p in precs for g in groups]
    calls += [("dequantize", *glu_sizes.W4_BACK, 0, p, 32) for p in precs]
    calls += [("empty", 0, 8, 6, 0, 0)]
    found = set().union(*(names(line) for line in launched(driver, calls)))
    every = names(run(driver, "all").stdout)
    assert len(every) > 100 and found == every, sorted(every - found)


def test_sums_are_divided_where_there_are_few_results(driver):
    """Sizes of the tests among them: the products' partial sums are added by a kernel of
    their own."""
    lines = launched(driver, [("grad", *s, 2, 0) for s in [(16_000, 128, 512), (1000, 100, 511), (16_384, 4096, 8192)]])
    assert ["dense_join" in line for line in lines] == [True, True, False]


# n, d, f, precision, group, and whether the kernel for few rows takes less time than
# tiles (us of both): they differ by a tenth or more.
FEW_ROWS = [
    (33, 4096, 8192, 2, 128, True),     # 20, 61
    (128, 4096, 8192, 2, 128, True),    # 38, 63
    (256, 4096, 8192, 2, 128, False),   # 73, 64
    (512, 4096, 8192, 2, 128, False),   # 142, 66
    (256, 1536, 1536, 2, 64, True),     # 10, 34
    (1000, 1536, 1536, 2, 64, True),    # 28, 35
    (128, 4096, 8192, 2, 32, True),     # 40, 103
    (512, 4096, 8192, 2, 32, False),    # 152, 109
    (64, 4096, 4096, 0, 128, True),     # 48, 97
    (512, 300, 500, 0, 32, True),       # 12, 18
]


def test_products_of_few_rows_take_the_faster_kernel(driver):
    lines = launched(driver, [("w4", *c[:5]) for c in FEW_ROWS])
    for c, line in zip(FEW_ROWS, lines):
        assert ("rows_kernel" in line) == c[5], (c, line)
