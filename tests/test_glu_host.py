"""The gated block and 4-bit weights on the host: the layout, the refusals of every
entry point of the C ABI and of the Python binding, and the 64-bit forms the GPU
tests compare with (CPU only)."""
import ctypes

import numpy as np
import pytest
import torch

import glu_reference as ref
from paper_2101_08763_amd import api

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails or stops first
ODD = ctypes.c_void_p(0x1008)
EINVAL, OK = api.EXEMCL_EINVAL, api.EXEMCL_OK


@pytest.fixture(scope="module")
def lib():
    return api.load()


def call(lib, name, order, good, bad):
    a = dict(good)
    a.update(bad)
    return getattr(lib, name)(*[a[k] for k in order.split()], None)


GLU = dict(x=FAKE, n=10, d=40, Wg=FAKE, Wu=FAKE, f=20, bg=None, bu=None, precision=0, act=0, h=FAKE, g=None, u=None)
GLU_ORDER = "x n d Wg Wu f bg bu precision act h g u"
BAD_GLU = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 20) + 1), dict(f=-1), dict(f=(1 << 20) + 1), dict(precision=3),
           dict(precision=-1), dict(act=-1), dict(act=4), dict(x=None), dict(Wg=None), dict(Wu=None), dict(h=None)]


@pytest.mark.parametrize("bad", BAD_GLU, ids=[str(b) for b in BAD_GLU])
def test_glu_refuses(lib, bad):
    assert call(lib, "exemplar_glu", GLU_ORDER, GLU, bad) == EINVAL


GRAD = dict(dh=FAKE, x=FAKE, Wg=FAKE, Wu=FAKE, g=FAKE, u=FAKE, n=10, d=40, f=20, precision=0, act=0, dx=FAKE, dWg=FAKE, dWu=FAKE,
            dbg=None, dbu=None)
GRAD_ORDER = "dh x Wg Wu g u n d f precision act dx dWg dWu dbg dbu"
BAD_GRAD = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 20) + 1), dict(f=-1), dict(f=(1 << 20) + 1), dict(precision=3),
            dict(act=4), dict(dh=None), dict(x=None), dict(Wg=None), dict(Wu=None), dict(g=None), dict(u=None)]


@pytest.mark.parametrize("bad", BAD_GRAD, ids=[str(b) for b in BAD_GRAD])
def test_glu_backward_refuses(lib, bad):
    assert call(lib, "exemplar_glu_backward", GRAD_ORDER, GRAD, bad) == EINVAL


def test_within_the_workspace_limit(lib, monkeypatch):
    monkeypatch.setenv("EXEMCL_WORKSPACE_LIMIT", "1024")
    assert call(lib, "exemplar_glu_backward", GRAD_ORDER, GRAD, dict(n=1000)) == api.EXEMCL_ENOMEM
    assert call(lib, "exemplar_glu", GLU_ORDER, GLU, dict(n=1000)) == api.EXEMCL_ENOMEM  # fp32: laid out again


QUANT = dict(w=FAKE, n=10, d=40, precision=0, group=32, codes=FAKE, words=FAKE)
BAD_QUANT = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(precision=3), dict(group=0), dict(group=16),
             dict(group=96), dict(group=256), dict(w=None), dict(codes=None), dict(words=None), dict(codes=ODD), dict(words=ODD)]


@pytest.mark.parametrize("bad", BAD_QUANT, ids=[str(b) for b in BAD_QUANT])
def test_w4_quantize_and_dequantize_refuse(lib, bad):
    assert call(lib, "exemplar_w4_quantize", "w n d precision group codes words", QUANT, bad) == EINVAL
    assert call(lib, "exemplar_w4_dequantize", "codes words n d group precision w", QUANT, bad) == EINVAL


PRODUCT = dict(x=FAKE, n=3, d=40, precision=0, codes=FAKE, words=FAKE, f=10, group=64, bias=None, y=FAKE)
PRODUCT_ORDER = "x n d precision codes words f group bias y"
BAD_PRODUCT = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(precision=3), dict(f=-1), dict(f=2**31),
               dict(group=48), dict(x=None), dict(codes=None), dict(words=None), dict(codes=ODD), dict(words=ODD), dict(y=None)]


@pytest.mark.parametrize("bad", BAD_PRODUCT, ids=[str(b) for b in BAD_PRODUCT])
def test_w4_product_refuses(lib, bad):
    assert call(lib, "exemplar_w4_product", PRODUCT_ORDER, PRODUCT, bad) == EINVAL


W4GLU = dict(x=FAKE, n=3, d=40, precision=0, gc=FAKE, gw=FAKE, uc=FAKE, uw=FAKE, f=10, group=64, bg=None, bu=None, act=0, h=FAKE)
W4GLU_ORDER = "x n d precision gc gw uc uw f group bg bu act h"
BAD_W4GLU = [dict(n=-1), dict(n=2**31), dict(d=0), dict(d=(1 << 22) + 1), dict(precision=3), dict(f=-1), dict(f=2**31),
             dict(group=48), dict(act=4), dict(act=-1), dict(x=None), dict(h=None),
             *(dict([(k, v)]) for k in ("gc", "gw", "uc", "uw") for v in (None, ODD))]


@pytest.mark.parametrize("bad", BAD_W4GLU, ids=[str(b) for b in BAD_W4GLU])
def test_w4_glu_refuses(lib, bad):
    assert call(lib, "exemplar_w4_glu", W4GLU_ORDER, W4GLU, bad) == EINVAL


def test_nothing_to_do(lib):
    assert call(lib, "exemplar_glu", GLU_ORDER, GLU, dict(n=0, x=None, h=None)) == OK
    assert call(lib, "exemplar_glu", GLU_ORDER, GLU, dict(f=0, Wg=None, Wu=None, h=None)) == OK
    none = dict(dx=None, dWg=None, dWu=None)
    assert call(lib, "exemplar_glu_backward", GRAD_ORDER, GRAD, none) == OK
    assert call(lib, "exemplar_glu_backward", GRAD_ORDER, GRAD, dict(n=0, dh=None, x=None, g=None, u=None, **none)) == OK
    assert call(lib, "exemplar_glu_backward", GRAD_ORDER, GRAD, dict(f=0, dh=None, g=None, u=None, Wg=None, Wu=None, **none)) == OK
    assert call(lib, "exemplar_w4_quantize", "w n d precision group codes words", QUANT, dict(n=0, w=None, codes=None, words=None)) == OK
    assert call(lib, "exemplar_w4_dequantize", "codes words n d group precision w", QUANT,
                dict(n=0, w=None, codes=None, words=None)) == OK
    assert call(lib, "exemplar_w4_product", PRODUCT_ORDER, PRODUCT, dict(n=0, x=None, y=None)) == OK
    assert call(lib, "exemplar_w4_product", PRODUCT_ORDER, PRODUCT, dict(f=0, codes=None, words=None, y=None)) == OK
    assert call(lib, "exemplar_w4_glu", W4GLU_ORDER, W4GLU, dict(n=0, x=None, h=None)) == OK
    assert call(lib, "exemplar_w4_glu", W4GLU_ORDER, W4GLU, dict(f=0, gc=None, gw=None, uc=None, uw=None, h=None)) == OK


@pytest.mark.parametrize("n,d,group,codes,words", [(0, 1, 32, 0, 0), (1, 1, 128, 1024, 16), (16, 128, 32, 1024, 64),
                                                   (17, 129, 64, 4096, 128), (4096, 1536, 128, 4096 * 768, 4096 * 12)])
def test_w4_layout(n, d, group, codes, words):
    assert api.exemplar_w4_layout(n, d, group) == (codes, words)


@pytest.mark.parametrize("bad", [(-1, 4, 32), (2**31, 4, 32), (4, 0, 32), (4, (1 << 22) + 1, 32), (4, 4, 16)])
def test_w4_layout_refuses(bad):
    with pytest.raises(api.ExemclError):
        api.exemplar_w4_layout(*bad)


def w4(n, d, group):
    tiles, blocks = -(-n // 16), -(-d // 128)
    return api.W4Rows(torch.zeros(tiles, blocks, 1024, dtype=torch.uint8),
                      torch.zeros(tiles, blocks * 128 // group, 16, dtype=torch.int32), n, d, group)


def test_binding_refuses():
    x, W, h = torch.zeros(4, 40), torch.zeros(20, 40), torch.zeros(4, 20)
    q = w4(20, 40, 32)
    glu, back = api.exemplar_glu, api.exemplar_glu_backward
    for f, error in (
            (lambda: glu(x, W, W), ValueError),                                # not on the GPU
            (lambda: glu(x[0], W, W), ValueError),
            (lambda: glu(x, W[0], W), ValueError),
            (lambda: glu(x.double(), W.double(), W.double()), TypeError),
            (lambda: glu(x, W.half(), W.half()), ValueError),
            (lambda: glu(x, W, W[:19]), ValueError),
            (lambda: glu(x, W[:, :39], W[:, :39]), ValueError),
            (lambda: glu(x, W, W, torch.zeros(19)), ValueError),
            (lambda: glu(x, W, W, None, torch.zeros(20).half()), ValueError),
            (lambda: glu(x, W, W, out=torch.zeros(4, 21)), ValueError),
            (lambda: glu(x, W, W, out=h.half()), ValueError),
            (lambda: back(h, x, W, W, h, h), ValueError),                      # not on the GPU
            (lambda: back(h[:3], x, W, W, h, h), ValueError),
            (lambda: back(h, x, W, W, h[:3], h), ValueError),
            (lambda: back(h, x, W, W, h, h.half()), ValueError),
            (lambda: back(h, x, W, W[:19], h, h), ValueError),
            (lambda: back(h, x[0], W, W, h, h), ValueError),
            (lambda: api.exemplar_w4_quantize(W), ValueError),                 # not on the GPU
            (lambda: api.exemplar_w4_quantize(W[0]), ValueError),
            (lambda: api.exemplar_w4_quantize(W, 48), ValueError),
            (lambda: api.exemplar_w4_quantize(W.double()), TypeError),
            (lambda: api.exemplar_w4_dequantize(q, torch.float64), TypeError),
            (lambda: api.exemplar_w4_dequantize(q._replace(d=200), torch.float32), ValueError),
            (lambda: api.exemplar_w4_dequantize(q._replace(n=33), torch.float32), ValueError),
            (lambda: api.exemplar_w4_dequantize(q._replace(group=64), torch.float32), ValueError),
            (lambda: api.exemplar_w4_dequantize(q._replace(group=20), torch.float32), ValueError),
            (lambda: api.exemplar_w4_dequantize(q._replace(codes=q.codes.int()), torch.float32), ValueError),
            (lambda: api.exemplar_w4_dequantize(q, torch.float32, out=torch.zeros(20, 41)), ValueError),
            (lambda: api.exemplar_w4_product(x, q), ValueError),               # not on the GPU
            (lambda: api.exemplar_w4_product(x[0], q), ValueError),
            (lambda: api.exemplar_w4_product(x[:, :39].contiguous(), q), ValueError),
            (lambda: api.exemplar_w4_product(x, q, bias=torch.zeros(19)), ValueError),
            (lambda: api.exemplar_w4_product(x, q, out=torch.zeros(4, 19)), ValueError),
            (lambda: api.exemplar_w4_glu(x, q, w4(19, 40, 32)), ValueError),
            (lambda: api.exemplar_w4_glu(x, q, w4(20, 40, 64)), ValueError),
            (lambda: api.exemplar_w4_glu(x, q, w4(20, 41, 32)), ValueError),
            (lambda: api.exemplar_w4_glu(x, q, q, torch.zeros(20).half()), ValueError),
            (lambda: api.exemplar_w4_glu(x, q, q), ValueError)):               # not on the GPU
        with pytest.raises(error):
            f()


# -- the 64-bit forms ----------------------------------------------------------
@pytest.mark.parametrize("act", ref.ACTIVATIONS)
def test_reference_gradient_by_differences(act):
    """The gradient's formula against central differences of the block's (64 bits,
    step 1e-6: their error is about 1e-12 / 1e-6 + 1e-12)."""
    r = torch.Generator().manual_seed(5)
    n, d, f = 3, 4, 5
    x, Wg, Wu, bg, bu, dh = (torch.randn(*s, dtype=torch.float64, generator=r)
                             for s in ((n, d), (f, d), (f, d), (f,), (f,), (n, f)))
    _, g, u = ref.glu(x, Wg, Wu, bg, bu, act)
    grads = ref.glu_backward(dh, x, Wg, Wu, g, u, act)
    leaves, step = [x, Wg, Wu, bg, bu], 1e-6
    for at, (leaf, grad) in enumerate(zip(leaves, grads)):
        for i in range(leaf.numel()):
            side = []
            for s in (step, -step):
                moved = [t.clone() for t in leaves]
                moved[at].view(-1)[i] += s
                side.append(float((ref.glu(*moved, act)[0] * dh).sum()))
            assert abs((side[0] - side[1]) / (2 * step) - float(grad.reshape(-1)[i])) < 1e-7


def test_reference_4_bits_by_hand():
    # s = 15 / 15, z = 5: ties to even, both ends
    w = np.zeros((1, 32), np.float32)
    w[0, :6] = [-5.0, 10.0, 0.5, 1.5, 2.4, -0.6]
    q, s, z = ref.w4_round(w, 32)
    assert s[0, 0] == 1 and z[0, 0] == 5
    assert ref.w4_values(q, s, z, 32)[0, :7].tolist() == [-5.0, 10.0, 0.0, 2.0, 2.0, -1.0, 0.0]
    # only positive values: z = 0; only zeros: s = 0; an infinity: NaN
    w[0] = 3.0
    q, s, z = ref.w4_round(w, 32)
    assert z[0, 0] == 0 and np.all(q == 15) and abs(15 * s[0, 0] / 3 - 1) < 2.0 ** -14 and 15 * s[0, 0] >= 3
    q, s, z = ref.w4_round(np.zeros((1, 32), np.float32), 32)
    assert s[0, 0] == 0 and np.all(ref.w4_values(q, s, z, 32) == 0)
    w[0, 7] = np.inf
    assert np.isnan(ref.w4_values(*ref.w4_round(w, 32), 32)).all()


@pytest.mark.parametrize("group", [32, 64, 128])
def test_reference_layout_there_and_back(group):
    g = np.random.default_rng(group)
    w = g.standard_normal((19, 200)).astype(np.float32)
    q, s, z = ref.w4_round(w, group)
    codes, words = ref.w4_store(q, s, z, group)
    assert (codes.nbytes, words.size) == api.exemplar_w4_layout(19, 200, group)
    assert np.array_equal(ref.w4_load(codes, words, 19, 200, group), ref.w4_values(q, s, z, group))
    # half a step, of a scale that is at most 2^-15 above the range's fifteenth
    assert np.all(np.abs(ref.w4_values(q, s, z, group) - w) <= 0.51 * np.repeat(s, group, 1)[:, :200])
