"""Forward-mode derivatives through the calls on rows, the gated block and 4-bit weights
(CPU only: checks come before the device's)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2101_08763_amd import api


def w4(n, d, group):
    tiles, blocks = -(-n // 16), -(-d // 128)
    return api.W4Rows(torch.zeros(tiles, blocks, 1024, dtype=torch.uint8),
                      torch.zeros(tiles, blocks * 128 // group, 16, dtype=torch.int32), n, d, group)


def mx(n, d, fmt):
    dp = (d + 127) // 128 * 128
    return api.MxRows(torch.zeros(n, dp * fmt // 8, dtype=torch.uint8), torch.zeros(n, dp // 32, dtype=torch.uint8), d, fmt)


X, W, F, H = torch.zeros(4, 40), torch.zeros(20, 40), torch.zeros(20), torch.zeros(4, 20)
CALLS = {
    "norm": (lambda x, w, r: api.exemplar_rmsnorm(x, w, r), (X, X[0], X)),
    "norm_backward": (lambda dy, h, w, s: api.exemplar_rmsnorm_backward(dy, h, w, s), (X, X, X[0], X[:, 0].clone())),
    "mx_product": (lambda bias: api.exemplar_mx_product(mx(4, 40, 8), mx(20, 40, 4), bias=bias), (F,)),
    "glu": (lambda *a: api.exemplar_glu(*a), (X, W, W, F, F)),
    "glu_backward": (lambda *a: api.exemplar_glu_backward(*a), (H, X, W, W, H, H)),
    "w4_product": (lambda x, b: api.exemplar_w4_product(x, w4(20, 40, 32), bias=b), (X, F)),
    "w4_glu": (lambda x, b, c: api.exemplar_w4_glu(x, w4(20, 40, 32), w4(20, 40, 32), b, c), (X, F, F)),
}


@pytest.mark.parametrize("name,at", [(name, at) for name, (_, args) in CALLS.items() for at in range(len(args))])
def test_a_tangent_is_not_lost_silently(name, at):
    call, args = CALLS[name]
    with forward_ad.dual_level():
        given = [forward_ad.make_dual(t, torch.ones_like(t)) if i == at else t for i, t in enumerate(args)]
        with pytest.raises(ValueError, match="forward-mode"):
            call(*given)
        with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):  # which leaves forward mode on
            call(*given)
        primals = [forward_ad.unpack_dual(t).primal for t in given]
        with pytest.raises(ValueError, match="on the GPU"):
            call(*primals)
    with pytest.raises(ValueError, match="on the GPU"):
        call(*args)


@pytest.mark.parametrize("name", CALLS)
def test_function_transforms_are_refused(name):
    """torch.func's tensors have no memory of their own to give."""
    call, args = CALLS[name]
    with pytest.raises(RuntimeError, match="data pointer"):
        torch.func.jvp(call, args, tuple(torch.ones_like(t) for t in args))


def test_rounding_weights_with_a_tangent():
    """Codes have no derivative: weights are rounded as they are."""
    with forward_ad.dual_level():
        w = forward_ad.make_dual(W, W)
        for call in (lambda: api.exemplar_w4_quantize(w), lambda: api.exemplar_mx_quantize(w, api.EXEMCL_MXFP4)):
            with pytest.raises(ValueError, match="on the GPU"):
                call()
