"""Tensors that require a gradient (CPU only: checks come before the device's)."""
import pytest
import torch

from paper_2101_08763_amd import api


def rows(n, d, fmt):
    dp = (d + 127) // 128 * 128
    return api.MxRows(torch.zeros(n, dp * fmt // 8, dtype=torch.uint8), torch.zeros(n, dp // 32, dtype=torch.uint8), d, fmt)


X, W, R, S = torch.zeros(4, 40), torch.zeros(40), torch.zeros(4, 40), torch.zeros(4)
CALLS = {
    "norm": (lambda x, w, r: api.exemplar_rmsnorm(x, w, r), (X, W, R)),
    "norm_rows": (lambda x, w, r: api.exemplar_rmsnorm(x, w, r, format=api.EXEMCL_MXFP8), (X, W, R)),
    "backward": (lambda dy, h, w, s, dh: api.exemplar_rmsnorm_backward(dy, h, w, s, dh=dh), (X, X, W, S, R)),
    "product": (lambda bias: api.exemplar_mx_product(rows(4, 40, 8), rows(4, 40, 4), bias=bias), (S,)),
}


@pytest.mark.parametrize("name,at", [(name, at) for name, (_, args) in CALLS.items() for at in range(len(args))])
def test_a_gradient_is_not_lost_silently(name, at):
    call, args = CALLS[name]
    given = [t.clone().requires_grad_(i == at) for i, t in enumerate(args)]
    with pytest.raises(ValueError, match="records no gradient"):
        call(*given)
    with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
        call(*given)
    with pytest.raises(ValueError, match="on the GPU"):
        call(*args)


def test_rounding_a_parameter():
    """Codes have no gradient: weights are rounded as they are."""
    with pytest.raises(ValueError, match="on the GPU"):
        api.exemplar_mx_quantize(X.clone().requires_grad_(), api.EXEMCL_MXFP4)
