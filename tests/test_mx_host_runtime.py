"""The host code of the calls on microscaled rows over a HIP runtime that
launches nothing (tests/fake_hip/mx_driver.cpp), without a GPU."""
import os
import re
import subprocess

import pytest

import mx_sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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
    tmp = tmp_path_factory.mktemp("fake_hip_mx")
    drv, exe = str(tmp / "driver.o"), str(tmp / "driver")
    for cmd in ([B.HIPCC, "-O1", "-std=c++17", f"-I{B.INCLUDE}", "-Wno-unused-value", "-Wno-unused-function", "-c",
                 os.path.join(ROOT, "tests", "fake_hip", "mx_driver.cpp"), "-o", drv],
                [B.HIPCC, f"--offload-arch={B.ARCH}", drv, *objs, "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stdout + r.stderr
    return exe


def run(driver, *args, stdin=""):
    env = {k: v for k, v in os.environ.items() if not k.startswith("EXEMCL_")}
    return subprocess.run([driver, *args], input=stdin, capture_output=True, text=True, timeout=300, env=env)


@pytest.mark.parametrize("check", ["capture", "members"])
def test_host_runtime(driver, check):
    r = run(driver, check)
    assert r.returncode == 0 and "checks passed" in r.stdout, r.stdout + r.stderr


def kernels(driver, calls):
    """Per call (name and up to five numbers) its kernels, as plain_name has them."""
    return [[k for k in map(plain_name, line.split()) if k] for line in run_calls(driver, calls)]


def run_calls(driver, calls):
    r = run(driver, "calls", stdin="".join(" ".join(map(str, (*c, 0, 0, 0)[:6])) + "\n" for c in calls))
    lines = r.stdout.splitlines()
    assert r.returncode == 0 and len(lines) == len(calls) + 1, r.stdout + r.stderr
    return lines[:-1]


def plain_name(symbol):
    """(name, element type, numbers) of a kernel on rows from "symbol:workgroups"."""
    m = re.search(r"\d((?:mx|rmsnorm|column)_[a-z0-9_]+?_kernel)(I(.*?)EEv)?", symbol)
    if not m:
        return None
    args = m.group(3) or ""
    kind = re.match(r"DF16b|DF16_|f", args)
    return (m.group(1), kind.group(0) if kind else "", *(int(x) for x in re.findall(r"L[ib](\d+)E", args + "E")))


def compiled(driver, name):
    """Every kernel of the library whose name starts so."""
    r = run(driver, "all")
    assert r.returncode == 0
    return {k for k in map(plain_name, r.stdout.split()) if k and k[0].startswith(name)}


# m, n, d, format of A, precision (0: fp32, 2: bf16), and whether 16 x 16 tiles
# take less time than 64 x 128 (us of both): the two differ by a tenth or more.
FEW_ROWS = [
    (1, 2000, 1024, 8, 2, True),     # 3.1, 11.0
    (1, 20_000, 1536, 4, 0, True),   # 6.1, 8.4
    (1, 20_000, 1536, 4, 2, True),   # 6.1, 8.1
    (1, 20_000, 1536, 8, 2, True),   # 6.8, 15.5
    (1, 28_672, 8192, 8, 0, True),   # 36.6, 64.5
    (1, 28_672, 8192, 8, 2, True),   # 36.6, 65.0
    (1, 50_000, 256, 8, 0, True),    # 5.1, 7.9
    (1, 50_000, 256, 4, 0, True),    # 4.7, 5.8
    (4, 28_672, 8192, 8, 2, True),   # 44.3, 65.8
    (8, 20_000, 1536, 4, 2, True),   # 7.1, 9.0
    (8, 28_672, 8192, 8, 2, True),   # 51.9, 66.1
    (16, 20_000, 1536, 4, 0, True),  # 8.4, 10.2
    (16, 50_000, 256, 8, 2, True),   # 6.7, 8.9
    (16, 28_672, 8192, 4, 2, False),  # 55.2, 36.6
    (24, 8192, 4096, 8, 2, True),    # 18.7, 34.0
    (24, 20_000, 1536, 4, 2, False),  # 12.3, 9.0
    (24, 28_672, 8192, 8, 2, False),  # 115, 66.4
    (48, 8192, 1024, 8, 2, True),    # 9.9, 12.3
    (48, 8192, 4096, 4, 2, False),   # 24.1, 14.8
    (48, 20_000, 1536, 8, 2, False),  # 23.3, 16.6
    (130, 8192, 1024, 8, 2, False),  # 23.3, 12.6
    (130, 8192, 1024, 4, 0, False),  # 19.6, 9.1
]


def test_products_of_few_rows_take_the_faster_kernel(driver):
    got = kernels(driver, [("product", *c[:5]) for c in FEW_ROWS])
    for c, (kernel,) in zip(FEW_ROWS, got):
        assert (kernel[0] == "mx_product_direct_kernel") == c[5], (c, kernel)


def test_sizes_of_products_take_every_kernel(driver):
    """A kernel that is compiled is run by the tests on the GPU, whatever the rule
    that chooses it."""
    calls = [("product", *size, fmt, prec) for size in mx_sizes.PRODUCTS for fmt in (4, 8) for prec in (0, 1, 2)]
    assert {k for found in kernels(driver, calls) for k in found} == compiled(driver, "mx_product")


def test_sizes_of_sets_take_every_kernel(driver):
    """As with products; and the batch kernels take several groups of 16 sets one
    after the other in a workgroup."""
    calls = [("sets", *size) for size in mx_sizes.SETS]
    found = kernels(driver, calls)
    # (few points do not fill mx_fold_kernel's rows: test_sets_on_many_points)
    assert {k for f in found for k in f} | {("mx_fold_kernel", "")} == compiled(driver, ("mx_sets", "mx_bias", "mx_fold"))
    several = set()
    for (n, d, l, k), line in zip(mx_sizes.SETS, run_calls(driver, calls)):
        for symbol in line.split():
            name = plain_name(symbol)
            if name and name[0] == "mx_sets_kernel":
                points, groups = name[3] * name[4] * 16, -(-l // 16)
                if int(symbol.split(":")[1]) < -(-n // points) * groups:
                    several.add(name)
    assert {k[2:5] for k in several} == {k[2:5] for k in compiled(driver, "mx_sets_kernel")}


def test_sizes_of_gradients_take_every_kernel(driver):
    calls = [("gradient", *size, prec) for size in mx_sizes.GRADIENTS for prec in (0, 1, 2)]
    every = compiled(driver, ("rmsnorm_grad", "rmsnorm_dw", "column_sum"))
    assert {k for found in kernels(driver, calls) for k in found} == every
    for (n, d), line in zip(mx_sizes.GRADIENTS, run_calls(driver, calls)[::3]):
        for symbol in line.split():
            kind = plain_name(symbol)
            if kind and kind[0] == "rmsnorm_grad_kernel":  # more rows than workgroups take at once
                assert n > int(symbol.split(":")[1]) * (256 // kind[2]), (n, d, symbol)


def test_sizes_of_norms_and_roundings_take_every_kernel(driver):
    from test_mx_gpu import NORM_SIZES
    norms = [("norm", n, d, prec, fmt) for n, d in NORM_SIZES for prec in (0, 1, 2) for fmt in (0, 4, 8)]
    assert {k for found in kernels(driver, norms) for k in found} == compiled(driver, "rmsnorm_kernel")
    there_and_back = [(way, n, d, prec, fmt) for way in ("quantize", "dequantize") for n, d in mx_sizes.ROUNDINGS
                      for prec in (0, 1, 2) for fmt in (4, 8)]
    every = compiled(driver, ("mx_quantize", "mx_dequantize"))
    assert {k for found in kernels(driver, there_and_back) for k in found} == every
