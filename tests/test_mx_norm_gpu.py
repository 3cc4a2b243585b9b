"""The norm to microscaled rows where a row's root, or a result, is not finite."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2101_08763_amd import api

pytestmark = pytest.mark.gpu
FP4, FP8 = api.EXEMCL_MXFP4, api.EXEMCL_MXFP8
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("weight", [True, False])
@pytest.mark.parametrize("fmt", [FP4, FP8])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [1, 31, 32, 100, 129, 200, 1000, 8200])
def test_padding_of_rows_that_are_nan(d, dtype, fmt, weight):
    """Codes past d are zeros and blocks past d not NaN, also in rows of NaN (a NaN
    in them, or zeros without eps)."""
    x = torch.ones(4, d, dtype=dtype, device="cuda")
    x[1], x[2, d // 2] = 0.0, float("nan")
    w = torch.ones(d, dtype=dtype, device="cuda") if weight else None
    q, _, _ = api.exemplar_rmsnorm(x, w, eps=0.0, format=fmt)
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    blocks = -(-d // 32)
    assert np.all(scales[1:3, :blocks] == 255) and not np.any(scales[[0, 3]] == 255)
    assert not scales[:, blocks:].any()
    assert not codes[:, -(-d * fmt // 8):].any()
    if fmt == FP4 and d % 2:
        assert not (codes[:, d // 2] >> 4).any()


@pytest.mark.parametrize("fmt", [FP4, FP8])
def test_results_past_the_range_of_fp32(fmt):
    """y past fp32's largest number is infinite, and its block NaN; up to there it
    is rounded as any other.  One coordinate of 64 is not zero: rstd = 8."""
    largest = float(np.finfo(np.float32).max)
    x = torch.zeros(3, 64, device="cuda")
    x[0, 5], x[1, 40], x[2, 5] = 1.0, -3.0, -1.0
    w = torch.ones(64, device="cuda")
    w[5], w[40] = largest / 4.0, largest / 8.0
    q, _, rstd = api.exemplar_rmsnorm(x, w, eps=0.0, format=fmt)
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    assert np.all(scales[[0, 2], 0] == 255) and np.all(scales[[0, 2], 1] == 0)
    want = np.zeros((1, 64))
    want[0, 40] = -largest
    c, s = ref.quantize(want, fmt)
    assert np.array_equal(scales[1], s[0])
    assert np.array_equal(ref.values(codes[1:2], scales[1:2], 64, fmt), ref.values(c, s, 64, fmt))
