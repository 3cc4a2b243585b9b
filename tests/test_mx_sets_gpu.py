"""Scores of sets on 4-bit rows by every kernel (mx_sizes.SETS), in values whose sums
are exact.

Elements are multiples of 1/2 under scales of 1/2 and 1, so a product is a multiple
of 2^-4 and a bias of 2^-5; a point's part of a score is at most half its own
squared norm, and a check says that 24 bits hold 32 of them.  What is left is the
rounding of sums of 1 024 points (many points) to 24 bits, their sum in 64, and the
result: 2^-22 of it."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import mx_sizes
from paper_2101_08763_amd import api

pytestmark = pytest.mark.gpu
FP4 = api.EXEMCL_MXFP4


def clustered(n, d, seed):
    """Rows of 4 bits that share two thirds of their elements with one of five,
    as MxRows and in 64 bits (on the GPU)."""
    g = torch.Generator("cuda").manual_seed(seed)

    def random(high, *shape):
        return torch.randint(0, high, shape, generator=g, device="cuda", dtype=torch.uint8)

    dp = ref.padded(d)
    codes = random(16, 5, dp)[random(5, n).long()]
    codes = torch.where(random(3, n, dp) == 0, random(16, n, dp), codes)
    codes[:, d:] = 0
    scales = 126 + random(2, n, dp // 32)
    t = ref.table(FP4)
    table = torch.as_tensor(np.concatenate([t, -t])).cuda()
    values = table[codes.int()] * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)
    return api.MxRows(codes[:, 0::2] + 16 * codes[:, 1::2], scales, d, FP4), values[:, :d].contiguous()


def scores(V, sets):
    """f in 64 bits, in the clamp form, a block of points at a time."""
    n, (l, k) = V.shape[0], sets.shape
    at = sets.clamp(min=0).flatten().long()
    half = 0.5 * (V * V).sum(1)
    assert float(half.max()) * 32 * 32 < 2.0 ** 24
    E, bias = V[at].t().contiguous(), torch.where(sets.flatten() >= 0, -half[at], -torch.inf)
    f = torch.zeros(l, dtype=torch.float64, device="cuda")
    for i in range(0, n, 20_000):
        f += (V[i:i + 20_000] @ E + bias).view(-1, l, k).amax(2).clamp(min=0).sum(0)
    return f * 2.0 / n


@pytest.mark.parametrize("empty", [0.0, 0.3])
@pytest.mark.parametrize("n,d,l,k", mx_sizes.SETS + [(131_111, 300, 40, 5)])
def test_every_set_kernel(n, d, l, k, empty):
    q, V = clustered(n, d, n + d)
    g = torch.Generator("cuda").manual_seed(l + k)
    sets = torch.randint(0, n, (l, k), generator=g, device="cuda", dtype=torch.int32)
    if empty:
        sets[torch.rand(l, k, generator=g, device="cuda") < empty] = -1
        sets[l // 2] = -1
    want = scores(V, sets)
    got = api.exemplar_mx_eval(q, sets)
    assert float(want.max()) > 0
    assert torch.all((got.double() - want).abs() <= 2.0 ** -22 * want)
    if empty:
        assert float(got[l // 2]) == 0.0
        sets[l - 1, 0], sets[0, k - 1] = n, -2  # not rows of V
        bad = api.exemplar_mx_eval(q, sets)
        assert bad[[0, l - 1]].isnan().all() and torch.equal(bad[1:-1], got[1:-1])
