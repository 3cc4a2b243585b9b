"""fp32 values whose parts are small numbers of bf16, on the GPU."""
import pytest
import torch

import glu_reference as ref
from paper_2101_08763_amd import api
from test_glu_gpu import close, gen, randn, w4_bounds

pytestmark = pytest.mark.gpu

# Parts count down to bf16's last place, 2^-133: nothing is lost of values from 2^-110 on,
# and half of that place at most of smaller ones.
STEP = 2.0 ** -134


@pytest.mark.parametrize("e", [-100, -110, -116, -124])
@pytest.mark.parametrize("n,d,f", [(5, 130, 70), (700, 130, 1300)])
def test_block_and_gradient(n, d, f, e):
    r = gen("small", n, e)
    sign = torch.where(torch.rand(n, d, generator=r, device="cuda") < 0.5, -1.0, 1.0)
    x = sign * (1 + torch.rand(n, d, generator=r, device="cuda")) * 2.0 ** e
    Wg, Wu = (randn(r, f, d) * 2.0 ** 100 for _ in range(2))
    lost = 0.0 if e >= -110 else STEP
    _, g, u = api.exemplar_glu(x, Wg, Wu, activation=api.EXEMCL_RELU, save=True)
    x64 = x.double()
    for got, W in ((g, Wg.double()), (u, Wu.double())):
        want = ref.times(x64, W)
        b = ref.project_bounds(x64, W, None, torch.float32) + lost * W.abs().sum(1)
        close(got, want, b + 2.0 ** -24 * want.abs())
    # dW = dg' x with the small values on the other side
    dh = randn(r, n, f) * 2.0 ** 100
    one = torch.ones(n, f, device="cuda")
    du = api.exemplar_glu_backward(dh, x, Wg, Wu, one, one, activation=api.EXEMCL_RELU)[2]
    dh64 = dh.double()
    want, size = ref.times(dh64.t().contiguous(), x64.t()), ref.times(dh64.abs().t().contiguous(), x64.abs().t())
    b = ref.sum_bound(n, torch.float32) * size + lost * dh64.abs().sum(0)[:, None]
    close(du, want, b + 2.0 ** -24 * want.abs())


@pytest.mark.parametrize("e", [-100, -110, -116, -124])
@pytest.mark.parametrize("n,d,f", [(5, 130, 70), (2900, 700, 1500)])
def test_w4_product(n, d, f, e):
    r = gen("small w4", n, e)
    x = (1 + torch.rand(n, d, generator=r, device="cuda")) * 2.0 ** e
    q = api.exemplar_w4_quantize(randn(r, f, d) * 2.0 ** 100, 64)
    W = torch.as_tensor(ref.w4_load(q.codes.cpu().numpy(), q.words.cpu().numpy(), f, d, 64)).cuda()
    lost = 0.0 if e >= -110 else STEP
    want, _, bound = w4_bounds(x.double(), W, q, None, torch.float32)
    # (the parts' products run on q and z apart, both up to 15 steps)
    s = W.abs().amax(1)
    close(api.exemplar_w4_product(x, q), want, bound + lost * 30 * d * s)
