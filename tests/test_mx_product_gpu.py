"""Products of microscaled rows whose sums are exact in 24 bits, in every order:
whatever the type of the result, it is the exact sum rounded once.

With outliers, elements of A are multiples of 2^-9, of B of 2^-1, and the
magnitudes of a result's terms add up to less than 2^12: no partial sum needs more
than 22 bits.  Otherwise a check says that it needs no more than 24.  So a sum in
fp32 rounds nothing in any order, and what is left is the rounding to the result's
type (to nearest, ties to even)."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import mx_sizes
from paper_2101_08763_amd import api

pytestmark = pytest.mark.gpu
FP4, FP8 = api.EXEMCL_MXFP4, api.EXEMCL_MXFP8
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def gen(*key):
    return np.random.default_rng([ord(c) for c in repr(key)])


def on_gpu(codes, d, fmt):
    """Rows of these codes (n x d, one a coordinate) under scales of 1."""
    n, dp = codes.shape[0], ref.padded(d)
    wide = np.zeros((n, dp), np.uint8)
    wide[:, :d] = codes
    if fmt == FP4:
        wide = wide[:, 0::2] + 16 * wide[:, 1::2]
    return api.MxRows(torch.as_tensor(wide).cuda(), torch.full((n, dp // 32), 127, dtype=torch.uint8, device="cuda"), d, fmt)


def signed(table):
    return np.concatenate([table, -table])


def outlier_codes(g, m, n, d):
    """8-bit codes of magnitudes 2^-6 to 2^-3 with +448 and -448 in two
    neighbouring coordinates of every 64, where B has twice the same 0.5: the
    large products cancel, and what is left is the small ones' sum."""
    t = ref.table(FP8)
    small = np.flatnonzero((t >= 2.0 ** -6) & (t < 2.0 ** -3))
    a = g.choice(small, (m, d)) + 128 * g.integers(0, 2, (m, d))
    b = g.choice([1, 2, 3], (n, d)) + 8 * g.integers(0, 2, (n, d))
    for start in range(0, d - 1, 64)[:8]:
        at = start + 2 * int(g.integers(0, min(32, (d - start) // 2)))
        a[:, at], a[:, at + 1] = 126, 254
        b[:, at], b[:, at + 1] = 1, 1
    return a.astype(np.uint8), b.astype(np.uint8)


def check(C, a, b, dtype, bias=None):
    """C against the exact sums of a and b (values), in 64 bits."""
    want = torch.as_tensor(a).cuda() @ torch.as_tensor(b).cuda().t().contiguous()
    if bias is not None:
        want = want + bias.double()
    assert torch.equal(C, want.float().to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,n,d", mx_sizes.PRODUCTS)
def test_outliers_lose_nothing(m, n, d, dtype):
    g = gen("outliers", m, n, d)
    ca, cb = outlier_codes(g, m, n, d)
    t8, t4 = np.concatenate([ref.table(FP8), [np.nan]]), ref.table(FP4)
    C = api.exemplar_mx_product(on_gpu(ca, d, FP8), on_gpu(cb, d, FP4), dtype=dtype)
    check(C, signed(t8)[ca], signed(t4)[cb], dtype)


def exact_rows(g, n, d, fmt):
    """Rows of elements within few binades under scales of 1/2, 1 and 2: values
    that are multiples of 2^-4, as MxRows and in 64 bits (on the GPU)."""
    t = ref.table(fmt)
    codes = g.choice(np.flatnonzero((t == 0) | ((t >= 0.5) & (t < 4.0))) if fmt == FP8 else 8, (n, d))
    if fmt == FP8:
        codes = np.where(codes == 0, 0, codes & ~1)  # two bits of mantissa: multiples of 2^-3
    codes = codes + (128 if fmt == FP8 else 8) * g.integers(0, 2, (n, d))
    q = on_gpu(codes.astype(np.uint8), d, fmt)
    scales = g.integers(126, 129, (n, ref.padded(d) // 32)).astype(np.uint8)
    scales[:, -(-d // 32):] = 0
    q.scales.copy_(torch.as_tensor(scales))
    table = signed(np.concatenate([t, [np.nan]]) if fmt == FP8 else t)
    unit = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, 1)[:, :d]
    return q, torch.as_tensor(table[codes] * unit).cuda()


def exact_product(a, b, bias):
    """a b^T + bias in 64 bits, after a check that 24 hold every partial sum."""
    size = a.abs() @ b.abs().t().contiguous() + bias.abs().double()
    assert float(size.max()) * 2.0 ** 6 < 2.0 ** 24
    return a @ b.t().contiguous() + bias.double()


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("fmt", [FP4, FP8])
@pytest.mark.parametrize("m,n,d", mx_sizes.PRODUCTS)
def test_every_result_of_every_tile(m, n, d, fmt, dtype, bias):
    """Bit for bit, every element: rows, columns, scales and bias at their places."""
    g = gen("tiles", m, n, d, fmt)
    (A, a), (B, b) = exact_rows(g, m, d, fmt), exact_rows(g, n, d, FP4)
    add = torch.as_tensor(g.integers(-64, 65, n) / 8.0, dtype=torch.float32, device="cuda")
    want = exact_product(a, b, add if bias else torch.zeros_like(add))
    out = torch.full((m * n + 64,), 7.0, dtype=dtype, device="cuda")
    C = api.exemplar_mx_product(A, B, bias=add if bias else None, dtype=dtype, out=out[:m * n].view(m, n))
    assert torch.equal(C, want.float().to(dtype))
    assert torch.equal(out[m * n:], torch.full((64,), 7.0, dtype=dtype, device="cuda"))  # nothing past it


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("fmt", [FP4, FP8])
@pytest.mark.parametrize("m,n,d", mx_sizes.PRODUCTS)
def test_nan_blocks_on_tiles(m, n, d, fmt, dtype):
    """A NaN block makes its row or column NaN, in the first and the last of them
    and in every step's scales; nothing else changes."""
    g = gen("nan tiles", m, n, d, fmt)
    (A, _), (B, _) = exact_rows(g, m, d, fmt), exact_rows(g, n, d, FP4)
    plain = api.exemplar_mx_product(A, B, dtype=dtype)
    rows = sorted({0, m // 2, m - 1}) if m > 1 else []
    cols = sorted({0, n // 3, n - 70, n - 1})
    blocks = -(-d // 32)
    for i, r in enumerate(rows):
        A.scales[r, (5 * i + 3) % blocks] = 255
    for i, c in enumerate(cols):
        B.scales[c, (7 * i + blocks - 1) % blocks] = 255
    got = api.exemplar_mx_product(A, B, dtype=dtype)
    nan = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    nan[rows], nan[:, cols] = True, True
    assert torch.equal(got.isnan(), nan)
    assert torch.equal(got[~nan], plain[~nan])


def test_parts_of_8_bit_rows_on_tiles():
    """Every pair of a large and a small element of A in neighbouring coordinates
    (16 bits and 32 bits of results), on tiles of 128 x 256."""
    g = gen("pairs of elements")
    m, n, d = 1031, 12_001, 128
    t = ref.table(FP8)
    small = np.flatnonzero((t > 0) & (t < 2.0))
    large = np.flatnonzero(t >= 2.0)
    ca = np.zeros((m, d), np.int64)
    ca[:, 5], ca[:, 6] = g.choice(large, m), g.choice(small, m)
    ca[:, 77] = ca[:, 5] + 128  # the large one again, with the other sign
    cb = np.zeros((n, d), np.int64)
    cb[:, 5] = cb[:, 77] = g.integers(1, 8, n)
    cb[:, 6] = g.integers(1, 16, n)
    a, b = torch.as_tensor(t[ca[:, 6]]).cuda(), torch.as_tensor(signed(ref.table(FP4))[cb[:, 6]]).cuda()
    want = a[:, None] * b[None, :]
    A, B = on_gpu(ca.astype(np.uint8), d, FP8), on_gpu(cb.astype(np.uint8), d, FP4)
    for dtype in (torch.float32, torch.bfloat16):
        assert torch.equal(api.exemplar_mx_product(A, B, dtype=dtype), want.float().to(dtype))
