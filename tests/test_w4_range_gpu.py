"""Products by 4-bit weights with large scales and any words past their end, on the GPU."""
import pytest
import torch

import glu_reference as ref
import glu_sizes
from paper_2101_08763_amd import api
from test_glu_gpu import TYPES, close, gen, randn, w4_bounds

pytestmark = pytest.mark.gpu


# of few rows, and of tiles (of two sizes that they end in)
PRODUCTS = [(1, 200, 60), (40, 200, 60), glu_sizes.W4_LARGE[0], glu_sizes.W4_LARGE[1]]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("size", PRODUCTS, ids=str)
def test_large_scales(size, t, group):
    """Scales up to 2^127 and zero points up to 255, whose product is past fp32's range
    where the sums with small rows are not."""
    n, d, f = size
    r = gen("large scales", size, str(t), group)
    tiles, blocks = -(-f // 16), -(-d // 128)
    codes = torch.randint(0, 256, (tiles, blocks, 1024), generator=r, device="cuda").to(torch.uint8)
    s = torch.ldexp(1 + torch.rand(tiles, blocks * 128 // group, 16, generator=r, device="cuda"),
                    torch.randint(118, 127, (tiles, blocks * 128 // group, 16), generator=r, device="cuda"))
    words = (s.view(torch.int32) & -256) | torch.randint(0, 256, s.shape, generator=r, device="cuda").to(torch.int32)
    q = api.W4Rows(codes, words, f, d, group)
    W = torch.as_tensor(ref.w4_load(codes.cpu().numpy(), words.cpu().numpy(), f, d, group)).cuda()
    x = (randn(r, n, d) * 2.0 ** -90).to(t)
    want, e, _ = w4_bounds(x.double(), W, q, None, t)
    assert bool(W.abs().max() > torch.finfo(torch.float32).max) and bool(want.float().isfinite().all())
    e = 9 * e  # 255 + 15 steps where w4_bounds has 30
    close(api.exemplar_w4_product(x, q), want, e + ref.half(t) * (want.abs() + e))
    # the block: |a(g) u| of two such sums is off by each one's error times the other
    h = api.exemplar_w4_glu(x, q, q, activation=api.EXEMCL_RELU)
    square = want.clamp(min=0) * want
    eh = 2 * e * (want.abs() + e)
    close(h, square, eh + ref.half(t) * (square + eh))


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("n", [3, 40, 6000])
def test_words_of_groups_past_the_end(n, t):
    """Groups wholly past d take no part, whatever their codes, zero points and finite
    scales; nor do codes past d."""
    d, f, group = 40, 700, 32
    r = gen("past the end", n, str(t))
    q = api.exemplar_w4_quantize(randn(r, f, d) / d ** 0.5, group)
    x = randn(r, n, d).to(t)
    want = api.exemplar_w4_product(x, q)
    codes, words = q.codes.clone(), q.words.clone()
    # row r's coordinate 32 j + 8 p + e in byte 256 p + 16 r + 4 j + e % 4
    byte = torch.arange(1024, device="cuda")
    p, j = byte // 256, byte % 16 // 4
    past = (32 * j + 8 * p >= d)
    codes[:, :, past] = torch.randint(0, 256, (codes.shape[0], 1, int(past.sum())), generator=r, device="cuda").to(torch.uint8)
    top = torch.full((words.shape[0], 2, 16), float.fromhex("0x1.fffep127"), device="cuda")
    words[:, 2:] = (top.view(torch.int32) & -256) | 255
    assert torch.equal(api.exemplar_w4_product(x, api.W4Rows(codes, words, f, d, group)), want)
