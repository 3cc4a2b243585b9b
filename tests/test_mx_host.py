"""Microscaled rows on the host: the layout, the refusals of every entry point
of the C ABI and of the Python binding, and the 64-bit forms the GPU tests
compare with (CPU only)."""
import ctypes

import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2101_08763_amd import api

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails or stops first
ODD = ctypes.c_void_p(0x1002)
EINVAL = api.EXEMCL_EINVAL


@pytest.fixture(scope="module")
def lib():
    return api.load()


def call(lib, name, order, good, bad):
    a = dict(good)
    a.update(bad)
    return getattr(lib, name)(*[a[k] for k in order.split()], None)


QUANT = dict(x=FAKE, n=10, d=40, precision=0, format=4, codes=FAKE, scales=FAKE)
BAD_ROWS = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(precision=3), dict(format=0), dict(format=5),
            dict(x=None), dict(codes=None), dict(scales=None), dict(codes=ODD), dict(scales=ODD)]


@pytest.mark.parametrize("bad", BAD_ROWS, ids=[str(b) for b in BAD_ROWS])
def test_quantize_and_dequantize_refuse(lib, bad):
    assert call(lib, "exemplar_mx_quantize", "x n d precision format codes scales", QUANT, bad) == EINVAL
    assert call(lib, "exemplar_mx_dequantize", "codes scales n d format precision x", QUANT, bad) == EINVAL


NORM = dict(x=FAKE, r=None, w=None, n=10, d=40, precision=0, eps=1e-6, format=4, h=None, y=FAKE, scales=FAKE, rstd=None)
BAD_NORM = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(format=0, d=(1 << 24) + 1), dict(precision=-1),
            dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(format=1), dict(x=None), dict(y=None),
            dict(scales=None), dict(y=ODD)]


@pytest.mark.parametrize("bad", BAD_NORM, ids=[str(b) for b in BAD_NORM])
def test_rmsnorm_refuses(lib, bad):
    assert call(lib, "exemplar_rmsnorm", "x r w n d precision eps format h y scales rstd", NORM, bad) == EINVAL


GRAD = dict(dy=FAKE, h=FAKE, w=None, rstd=FAKE, dh=None, n=10, d=40, precision=0, dx=FAKE, dw=FAKE)
BAD_GRAD = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 24) + 1), dict(precision=3), dict(dy=None), dict(h=None),
            dict(rstd=None), dict(dx=None)]


@pytest.mark.parametrize("bad", BAD_GRAD, ids=[str(b) for b in BAD_GRAD])
def test_rmsnorm_backward_refuses(lib, bad):
    assert call(lib, "exemplar_rmsnorm_backward", "dy h w rstd dh n d precision dx dw", GRAD, bad) == EINVAL


def test_rmsnorm_backward_within_the_workspace_limit(lib, monkeypatch):
    monkeypatch.setenv("EXEMCL_WORKSPACE_LIMIT", "1024")
    assert call(lib, "exemplar_rmsnorm_backward", "dy h w rstd dh n d precision dx dw", GRAD,
                dict(n=10_000, d=1000)) == api.EXEMCL_ENOMEM


PRODUCT = dict(A=FAKE, As=FAKE, m=3, fa=8, B=FAKE, Bs=FAKE, n=10, d=40, bias=None, precision=0, C=FAKE)
BAD_PRODUCT = [dict(m=-1), dict(m=2**31), dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(fa=0), dict(fa=3),
               dict(precision=3), dict(A=None), dict(As=None), dict(B=None), dict(Bs=None), dict(C=None), dict(A=ODD),
               dict(As=ODD), dict(B=ODD), dict(Bs=ODD)]


@pytest.mark.parametrize("bad", BAD_PRODUCT, ids=[str(b) for b in BAD_PRODUCT])
def test_product_refuses(lib, bad):
    assert call(lib, "exemplar_mx_product", "A As m fa B Bs n d bias precision C", PRODUCT, bad) == EINVAL


EVAL = dict(codes=FAKE, scales=FAKE, n=100, d=40, sets=FAKE, l=4, k=3, out=FAKE)
BAD_EVAL = [dict(codes=None), dict(scales=None), dict(n=0), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(l=-1),
            dict(k=-1), dict(sets=None), dict(out=None), dict(codes=ODD), dict(scales=ODD)]


@pytest.mark.parametrize("bad", BAD_EVAL, ids=[str(b) for b in BAD_EVAL])
def test_eval_refuses(lib, bad):
    assert call(lib, "exemplar_mx_eval", "codes scales n d sets l k out", EVAL, bad) == EINVAL


def test_eval_within_the_workspace_limit(lib, monkeypatch):
    monkeypatch.setenv("EXEMCL_WORKSPACE_LIMIT", "1024")
    assert call(lib, "exemplar_mx_eval", "codes scales n d sets l k out", EVAL, dict(n=100_000)) == api.EXEMCL_ENOMEM


def test_nothing_to_do(lib):
    none = dict(x=None, codes=None, scales=None, n=0)
    assert call(lib, "exemplar_mx_quantize", "x n d precision format codes scales", QUANT, none) == api.EXEMCL_OK
    assert call(lib, "exemplar_mx_dequantize", "codes scales n d format precision x", QUANT, none) == api.EXEMCL_OK
    assert call(lib, "exemplar_rmsnorm", "x r w n d precision eps format h y scales rstd", NORM,
                dict(n=0, x=None, y=None, scales=None)) == api.EXEMCL_OK
    assert call(lib, "exemplar_rmsnorm_backward", "dy h w rstd dh n d precision dx dw", GRAD,
                dict(n=0, dy=None, h=None, rstd=None, dx=None, dw=None)) == api.EXEMCL_OK
    order = "A As m fa B Bs n d bias precision C"
    assert call(lib, "exemplar_mx_product", order, PRODUCT, dict(m=0, A=None, As=None, C=None)) == api.EXEMCL_OK
    assert call(lib, "exemplar_mx_product", order, PRODUCT, dict(n=0, B=None, Bs=None, C=None)) == api.EXEMCL_OK
    assert call(lib, "exemplar_mx_eval", "codes scales n d sets l k out", EVAL, dict(l=0, sets=None, out=None)) == api.EXEMCL_OK


@pytest.mark.parametrize("d,fp4,fp8,scales", [(1, 64, 128, 4), (128, 64, 128, 4), (129, 128, 256, 8), (1536, 768, 1536, 48),
                                              (1 << 22, 1 << 21, 1 << 22, 1 << 17)])
def test_layout(d, fp4, fp8, scales):
    assert api.exemplar_mx_layout(d, api.EXEMCL_MXFP4) == (fp4, scales)
    assert api.exemplar_mx_layout(d, api.EXEMCL_MXFP8) == (fp8, scales)
    for bad in ((0, 4), ((1 << 22) + 1, 4), (8, 0), (8, 6)):
        with pytest.raises(api.ExemclError):
            api.exemplar_mx_layout(*bad)


def rows(n, d, fmt):
    dp = ref.padded(d)
    return api.MxRows(torch.zeros(n, dp * fmt // 8, dtype=torch.uint8), torch.zeros(n, dp // 32, dtype=torch.uint8), d, fmt)


def test_binding_refuses():
    x = torch.zeros(4, 40)
    q4, q8 = rows(4, 40, 4), rows(4, 40, 8)
    sets = torch.zeros(2, 3, dtype=torch.int32)
    for f, error in (
            (lambda: api.exemplar_mx_quantize(x, 4), ValueError),                       # not on the GPU
            (lambda: api.exemplar_mx_quantize(x[0], 4), ValueError),
            (lambda: api.exemplar_mx_quantize(x.double(), 4), TypeError),
            (lambda: api.exemplar_mx_quantize(x, 6), ValueError),
            (lambda: api.exemplar_mx_quantize(x, 4, out=q8), ValueError),
            (lambda: api.exemplar_mx_quantize(x, 4, out=rows(5, 40, 4)), ValueError),
            (lambda: api.exemplar_mx_dequantize(q4, torch.float64), TypeError),
            (lambda: api.exemplar_mx_dequantize(q4._replace(d=200), torch.float32), ValueError),
            (lambda: api.exemplar_mx_dequantize(q4._replace(scales=q4.scales[:3]), torch.float32), ValueError),
            (lambda: api.exemplar_mx_dequantize(q4._replace(codes=q4.codes.int()), torch.float32), ValueError),
            (lambda: api.exemplar_rmsnorm(x[0]), ValueError),
            (lambda: api.exemplar_rmsnorm(x, weight=torch.zeros(41)), ValueError),
            (lambda: api.exemplar_rmsnorm(x, weight=torch.zeros(40).half()), ValueError),
            (lambda: api.exemplar_rmsnorm(x, residual=x[:3]), ValueError),
            (lambda: api.exemplar_rmsnorm(x, format=5), ValueError),
            (lambda: api.exemplar_rmsnorm_backward(x, x[:3], None, torch.zeros(3)), ValueError),
            (lambda: api.exemplar_rmsnorm_backward(x, x, None, torch.zeros(4).half()), ValueError),
            (lambda: api.exemplar_rmsnorm_backward(x, x, torch.zeros(39), torch.zeros(4)), ValueError),
            (lambda: api.exemplar_rmsnorm_backward(x, x, None, torch.zeros(4), dh=x.half()), ValueError),
            (lambda: api.exemplar_mx_product(q4, q8), ValueError),                      # B of 8 bits
            (lambda: api.exemplar_mx_product(q4, rows(4, 41, 4)), ValueError),
            (lambda: api.exemplar_mx_product(q4, q4, bias=torch.zeros(3)), ValueError),
            (lambda: api.exemplar_mx_product(q4, q4, dtype=torch.int32), TypeError),
            (lambda: api.exemplar_mx_product(q4, q4, out=torch.zeros(4, 5)), ValueError),
            (lambda: api.exemplar_mx_product(q4, q4), ValueError),                      # not on the GPU
            (lambda: api.exemplar_mx_eval(q8, sets), ValueError),
            (lambda: api.exemplar_mx_eval(q4, sets.long()), TypeError),
            (lambda: api.exemplar_mx_eval(q4, sets[0]), ValueError),
            (lambda: api.exemplar_mx_eval(q4, sets, out=torch.zeros(3)), ValueError)):
        with pytest.raises(error):
            f()


# -- the 64-bit forms ----------------------------------------------------------
def test_reference_rounding_by_hand():
    # 4 bits, scale 1 (largest magnitude 4): ties to even, saturation, signs
    x = np.zeros((1, 32))
    x[0, :10] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.2500001, 5.0, 7.9]
    codes, scales = ref.quantize(x, ref.FP4)
    assert scales[0].tolist() == [127, 0, 0, 0]
    assert ref.values(codes, scales, 10, ref.FP4)[0].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, -0.5, 4.0, 6.0]
    # 8 bits, scale 1 (largest magnitude 256)
    x[0, :7] = [256.0, 500.0, 17.0, 19.0, 2.0 ** -10, 2.0 ** -10 * 1.001, -3 * 2.0 ** -10]
    x[0, 7:] = 0
    codes, scales = ref.quantize(x, ref.FP8)
    assert scales[0, 0] == 127
    assert ref.values(codes, scales, 7, ref.FP8)[0].tolist() == [256.0, 448.0, 16.0, 20.0, 0.0, 2.0 ** -9, -2.0 ** -8]


@pytest.mark.parametrize("weight,stream", [(True, True), (False, False)])
def test_reference_gradient_by_differences(weight, stream):
    """The gradient's formula against central differences of the norm's (64
    bits, step 1e-6: their error is about 1e-12 / 1e-6 + 1e-12)."""
    g = np.random.default_rng(5)
    n, d, eps = 3, 7, 1e-3
    x, r, dy, dh = (g.standard_normal((n, d)) for _ in range(4))
    w = 1 + 0.3 * g.standard_normal(d) if weight else None
    dh = dh if stream else None

    def loss(x, w):
        y, v, _ = ref.rmsnorm(x, w, r, eps)
        return (y * dy).sum() + (0.0 if dh is None else (v * dh).sum())

    _, v, rstd = ref.rmsnorm(x, w, r, eps)
    dx, dw = ref.rmsnorm_backward(dy, v, w, rstd, dh)
    step = 1e-6
    for i in range(n):
        for j in range(d):
            e = np.zeros((n, d))
            e[i, j] = step
            assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - dx[i, j]) < 1e-7
    for j in range(d):
        e = np.zeros(d)
        e[j] = step
        base = np.ones(d) if w is None else w
        assert abs((loss(x, base + e) - loss(x, base - e)) / (2 * step) - dw[j]) < 1e-7


def test_reference_sets_are_the_oracles(oracle_lib):
    g = np.random.default_rng(6)
    V = g.standard_normal((40, 9))
    sets = g.integers(0, 40, (6, 4)).astype(np.int32)
    assert np.allclose(ref.f_of_sets(V, sets), oracle_lib.eval(V, sets), rtol=1e-12, atol=1e-12)
