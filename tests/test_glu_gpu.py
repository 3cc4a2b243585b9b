"""The gated block, its gradient and 4-bit weights on the GPU, against their 64-bit
forms on the same (rounded) inputs."""
import importlib.util
import pathlib
import zlib

import numpy as np
import pytest
import torch

import glu_reference as ref
import glu_sizes
from paper_2101_08763_amd import api

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = {"silu": api.EXEMCL_SILU, "gelu": api.EXEMCL_GELU, "gelu_tanh": api.EXEMCL_GELU_TANH, "relu": api.EXEMCL_RELU}
# every activation at some sizes, the first at all
ACT_OF = {i: ref.ACTIVATIONS[i % 4] for i in range(len(glu_sizes.GLU))}


def gen(*key):
    g = torch.Generator("cuda")
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def among_nan(t, shift=1):
    """t in memory that has NaN before and after it, `shift` elements past an
    alignment of 256 bytes."""
    flat = torch.full((t.numel() + 512 + shift,), float("nan"), dtype=t.dtype, device=t.device)
    out = flat[256 + shift:256 + shift + t.numel()].view(t.shape)
    return out.copy_(t)


def inside(shape, dtype, shift=0):
    """(buffer, view): a view of a buffer of sevens."""
    flat = torch.full((int(np.prod(shape)) + 512 + shift,), 7.0, dtype=dtype, device="cuda")
    return flat, flat[256 + shift:flat.numel() - 256].view(shape)


def untouched(flat, shift=0):
    return bool((flat[:256 + shift] == 7).all()) and bool((flat[-256:] == 7).all())


def close(got, want, bound, name=""):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: got {got[i].item()}, want "
                             f"{want[i].item()}, bound {bound[i].item()}")


def block(g, n, d, f, t, bias):
    x, Wg, Wu = randn(g, n, d).to(t), (randn(g, f, d) / d ** 0.5).to(t), (randn(g, f, d) / d ** 0.5).to(t)
    return x, Wg, Wu, (0.3 * randn(g, f) if bias else None), (0.3 * randn(g, f) if bias else None)


def wide(*ts):
    return [None if t is None else t.double() for t in ts]


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("at,size", list(enumerate(glu_sizes.GLU)), ids=str)
def test_glu(at, size, t):
    n, d, f = size
    bias, act = at % 3 != 0, ACT_OF[at]
    args = block(gen("glu", size, str(t)), n, d, f, t, bias)
    # odd places in memory every other time
    x, Wg, Wu = (among_nan(a, at % 2) for a in args[:3])
    flat, out = inside((n, f), t, at % 2)
    h, g, u = api.exemplar_glu(x, Wg, Wu, *args[3:], activation=ACTS[act], save=True, out=out)
    want = ref.glu(*wide(*args), act)
    for got, w, b, name in zip((h, g, u), want, ref.glu_bounds(*wide(*args), act, t), "hgu"):
        close(got, w, b, name)
    assert h is out and untouched(flat, at % 2)
    alone, none, _ = api.exemplar_glu(x, Wg, Wu, *args[3:], activation=ACTS[act])
    assert torch.equal(alone, h) and none is None  # without g and u, and again: the same bits


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("at,size", list(enumerate(glu_sizes.GLU)), ids=str)
def test_glu_backward(at, size, t):
    n, d, f = size
    act = ACT_OF[at]
    r = gen("backward", size, str(t))
    x, Wg, Wu, _, _ = block(r, n, d, f, t, False)
    dh, g, u = (0.5 * randn(r, n, f)).to(t), (1.5 * randn(r, n, f)).to(t), randn(r, n, f).to(t)
    g.view(-1)[::5] = 0.0  # relu's corner
    args = (dh, x, Wg, Wu, g, u)
    moved = [among_nan(a, at % 2) for a in args]
    got = api.exemplar_glu_backward(*moved, activation=ACTS[act], bias=True)
    want, bounds = ref.glu_backward(*wide(*args), act), ref.backward_bounds(*wide(*args), act, t)
    for a, w, b, name in zip(got, want, bounds, ("dx", "dWg", "dWu", "dbg", "dbu")):
        close(a, w, b, name)
    again = api.exemplar_glu_backward(*moved, activation=ACTS[act])
    assert all(torch.equal(a, b) for a, b in zip(got[:3], again[:3])) and again[3] is None and again[4] is None


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", glu_sizes.LARGE, ids=str)
def test_large_tiles(size, t):
    n, d, f = size
    r = gen("large", size, str(t))
    args = block(r, n, d, f, t, True)
    h, g, u = api.exemplar_glu(*args, save=True)
    for got, w, b, name in zip((h, g, u), ref.glu(*wide(*args), "silu"), ref.glu_bounds(*wide(*args), "silu", t), "hgu"):
        close(got, w, b, name)
    dh = randn(r, n, f).to(t)
    back = (dh, *args[:3], g, u)
    got = api.exemplar_glu_backward(*back, bias=True)
    for a, w, b, name in zip(got, ref.glu_backward(*wide(*back), "silu"), ref.backward_bounds(*wide(*back), "silu", t),
                             ("dx", "dWg", "dWu", "dbg", "dbu")):
        close(a, w, b, name)


@pytest.mark.parametrize("n", [40, 300])
def test_fp32_is_as_good_as_fp32(n):
    """Bounds for each element allow for chance; together they tell whether a product
    of parts is missing.  8 steps' roundings of half a unit for 32 products, of sums
    that are as large as the result on average: 2^-25 sqrt(8 * 301 / 32 * 6) = 2^-20.6
    of the result's root mean square with all six, and 2^-18.5 in place of a missing
    (hi, lo) (2^-18 / sqrt 3 of each factor)."""
    args = block(gen("parts", n), n, 301, 200, torch.float32, False)
    _, g, u = api.exemplar_glu(*args, save=True)
    _, wg, wu = ref.glu(*wide(*args), "silu")
    for got, want in ((g, wg), (u, wu)):
        assert float((got.double() - want).square().mean().sqrt() / want.square().mean().sqrt()) < 2.0 ** -20.6


def test_gradient_by_differences():
    """fp32 gradients against differences of the GPU's own h in fp32, summed in 64
    bits.  Two central differences, of steps s = 2^-6 and 2 s, as (4 D(s) - D(2 s)) / 3:
    one alone is off by s^2 / 6 times the third derivative, a sum over 70 rows of
    terms like dh u x^3 times a third derivative of up to 0.8 (x^3 is 1.6 on average,
    and up to 27): 1e-3 where they agree in sign.  Together the s^2 terms cancel, and
    s^4 / 30 times the fifth is left, 70 * 6 * 10 * 2e-9 = 8e-6.  Rounding: 350
    results, each off by about 2^-22 of chance, over s: sqrt(350) 2^-22 (4 / 3 + 1 / 6) /
    (2 s) = 2e-4."""
    n, d, f, step = 70, 6, 5, 2.0 ** -6
    r = gen("differences")
    leaves = list(block(r, n, d, f, torch.float32, True))
    dh = randn(r, n, f)
    _, g, u = api.exemplar_glu(*leaves, activation=ACTS["gelu"], save=True)
    grads = api.exemplar_glu_backward(dh, *leaves[:3], g, u, activation=ACTS["gelu"], bias=True)

    def difference(at, i, step):
        side = []
        for s in (step, -step):
            moved = [t.clone() for t in leaves]
            moved[at].view(-1)[i] += s
            side.append((float((api.exemplar_glu(*moved, activation=ACTS["gelu"])[0].double() * dh.double()).sum()),
                         float(moved[at].view(-1)[i])))
        return (side[0][0] - side[1][0]) / (side[0][1] - side[1][1])

    for at, i in [(0, 3), (0, 200), (1, 0), (1, 17), (2, 5), (2, 29), (3, 0), (3, 4), (4, 2)]:
        want = (4 * difference(at, i, step) - difference(at, i, 2 * step)) / 3
        assert abs(float(grads[at].view(-1)[i]) - want) <= 1e-3 * max(1.0, abs(want)), (at, i)


@pytest.mark.parametrize("n", [5, 200])
@pytest.mark.parametrize("t", TYPES, ids=str)
def test_nan_stays_in_its_row_and_column(n, t):
    """A row of x with a NaN makes its own results NaN, a weight's row its column;
    all others are as without them."""
    d, f = 200, 150
    r = gen("nan", n, str(t))
    x, Wg, Wu, _, _ = block(r, n, d, f, t, False)
    clean, g, u = api.exemplar_glu(x, Wg, Wu, save=True)
    bx, bw = x.clone(), Wu.clone()
    bx[3, 7], bw[11, d - 1] = float("nan"), float("nan")
    h, _, _ = api.exemplar_glu(bx, Wg, bw)
    nan = torch.zeros(n, f, dtype=torch.bool, device="cuda")
    nan[3], nan[:, 11] = True, True
    assert torch.equal(h.isnan(), nan) and torch.equal(h[~nan], clean[~nan])
    # the gradient: dh's row reaches its row of dx, and its column both weights' rows
    dh = randn(r, n, f).to(t)
    clean = api.exemplar_glu_backward(dh, x, Wg, Wu, g, u, bias=True)
    dh[3, 11] = float("nan")
    got = api.exemplar_glu_backward(dh, x, Wg, Wu, g, u, bias=True)
    for at, (a, b) in enumerate(zip(got, clean)):
        nan = torch.zeros_like(a, dtype=torch.bool)
        nan[3 if at == 0 else 11] = True
        assert torch.equal(a.isnan(), nan) and torch.equal(a[~nan], b[~nan])


@pytest.mark.parametrize("n,d,f", [(3, 70, 40), (700, 130, 1300)])
def test_rows_at_the_end_of_fp32(n, d, f):
    """Values that round to an infinity of the parts' type, or to its largest number,
    are whole in three parts: the bounds of any others hold."""
    r = gen("end", n)
    x, Wg, Wu, _, _ = block(r, n, d, f, torch.float32, False)
    x = x * 2.0 ** 123
    top = torch.finfo(torch.float32).max
    x[0, :6] = torch.tensor([top, -top, float.fromhex("0x1.fefffep127"), float.fromhex("0x1.ffp127"),
                             float.fromhex("-0x1.fep127"), float.fromhex("0x1.feffffp127")])
    Wg, Wu = Wg * 2.0 ** -90, Wu * 2.0 ** -90
    assert bool(x.isfinite().all())
    got = api.exemplar_glu(x, Wg, Wu, activation=api.EXEMCL_RELU, save=True)
    want = ref.glu(x.double(), Wg.double(), Wu.double(), None, None, "relu")
    for a, b, e, name in zip(got, want, ref.glu_bounds(x.double(), Wg.double(), Wu.double(), None, None, "relu", torch.float32), "hgu"):
        close(a, b, e, name)


@pytest.mark.parametrize("act", ref.ACTIVATIONS)
@pytest.mark.parametrize("t", TYPES, ids=str)
def test_activations_far_out(act, t):
    """g from -10^30 to 10^30 (fp16: 6 10^4) and at infinities: x and u are 1, so h is
    a(g), and dg is a'(g) for dh = 1."""
    top = 6e4 if t == torch.float16 else 1e30
    far = torch.logspace(-3, np.log10(top), 60, dtype=torch.float64)
    g = torch.cat((far, -far, torch.tensor([0.0, float("inf"), -float("inf")], dtype=torch.float64))).cuda().to(t)
    f = g.numel()
    one = torch.ones(1, f, dtype=t, device="cuda")
    W = torch.ones(f, 1, dtype=t, device="cuda")
    h, _, _ = api.exemplar_glu(torch.ones(1, 1, dtype=t, device="cuda"), g[:, None].contiguous(), W, activation=ACTS[act])
    want, slope = ref.activation(act, g.double())
    want[-2], want[-1], slope[-2], slope[-1] = float("inf"), 0.0, 1.0, 0.0
    size = g.double().abs().nan_to_num(posinf=0.0)
    finite = want.abs() < torch.finfo(t).max
    finite[-1] = False
    bound = half(t) * want.abs() + size * ref.act_bound(t) * (want != 0) + ref.TINY[t]
    close(h[0][finite], want[finite], bound[finite], "a")
    if t != torch.float32:  # an infinite weight of fp32 may make a NaN of its parts' products
        assert h[0, -2] == float("inf") and h[0, -1] == 0
    bg = torch.zeros(f, device="cuda")
    bg[-2:] = g[-2:].float()
    h, _, _ = api.exemplar_glu(torch.ones(1, 1, dtype=t, device="cuda"), torch.zeros_like(W), W, bg, activation=ACTS[act])
    assert h[0, -2] == float("inf") and h[0, -1] == 0 and bool((h[0, :-2] == 0).all())
    dbg = api.exemplar_glu_backward(one, torch.ones(1, 1, dtype=t, device="cuda"), W, W, g[None], one, activation=ACTS[act],
                                    bias=True)[3]
    close(dbg, slope, torch.full_like(slope, 64 * ref.act_bound(t)), "slope")


half = ref.half


@pytest.mark.parametrize("n", [3, 100])
def test_subnormal_fp16(n):
    """Numbers below 2^-14 count with all their bits: weights of k 2^-24 times rows of
    1024 (sums of k, exactly), and rows of k 2^-24 times weights of 1024."""
    d, f, t = 64, 48, torch.float16
    r = gen("subnormal", n)
    k = torch.randint(-500, 500, (f, d), generator=r, device="cuda")
    W = (k.double() * 2.0 ** -24).to(t)
    x = torch.full((n, d), 1024.0, dtype=t, device="cuda")
    _, g, u = api.exemplar_glu(x, W, W, save=True)
    want = (k.sum(1).double() * 2.0 ** -14)[None].expand(n, f)
    assert torch.equal(g.double(), want.to(t).double()) and torch.equal(u, g)
    kx = torch.randint(-500, 500, (n, d), generator=r, device="cuda")
    q = api.exemplar_w4_quantize(torch.full((f, d), 1024.0, device="cuda"), 32)
    values = api.exemplar_w4_dequantize(q, torch.float32).double()
    y = api.exemplar_w4_product((kx.double() * 2.0 ** -24).to(t), q)
    want = ref.times(kx.double() * 2.0 ** -24, values)
    close(y, want, 2.0 ** -11 * want.abs() + 2.0 ** -24)


def test_empty():
    x, W = torch.ones(0, 8, device="cuda"), torch.ones(6, 8, device="cuda")
    h, g, u = api.exemplar_glu(x, W, W, save=True)
    assert h.shape == g.shape == u.shape == (0, 6)
    dx, dWg, dWu, dbg, dbu = api.exemplar_glu_backward(h, x, W, W, g, u, bias=True)
    assert dx.shape == (0, 8) and all(bool((a == 0).all()) for a in (dWg, dWu, dbg, dbu)) and dWg.shape == (6, 8)
    x, W = torch.ones(3, 8, device="cuda").half(), torch.ones(0, 8, device="cuda").half()
    h, g, u = api.exemplar_glu(x, W, W, save=True)
    dx, dWg, dWu, dbg, dbu = api.exemplar_glu_backward(h, x, W, W, g, u, bias=True)
    assert bool((dx == 0).all()) and dx.shape == (3, 8) and dWg.shape == (0, 8) and dbg.shape == (0,)


def test_parts_of_the_gradient():
    """Each output alone has the bits it has among all, through the C ABI."""
    n, d, f, t = 150, 72, 90, torch.bfloat16
    r = gen("parts of the gradient")
    x, Wg, Wu, _, _ = block(r, n, d, f, t, False)
    dh, g, u = (randn(r, n, f).to(t) for _ in range(3))
    every = api.exemplar_glu_backward(dh, x, Wg, Wu, g, u, bias=True)
    for at in range(5):
        out = torch.full_like(every[at], 7.0)
        ptrs = [out.data_ptr() if i == at else None for i in range(5)]
        rc = api.load().exemplar_glu_backward(dh.data_ptr(), x.data_ptr() if at in (1, 2) else None,
                                              Wg.data_ptr() if at == 0 else None, Wu.data_ptr() if at == 0 else None,
                                              g.data_ptr(), u.data_ptr(), n, d, f, api.EXEMCL_BF16, 0, *ptrs, None)
        torch.cuda.synchronize()
        assert rc == api.EXEMCL_OK and torch.equal(out, every[at]), at


# -- 4-bit weights -------------------------------------------------------------------
def weights(g, f, d, group, spread=True):
    w = randn(g, f, d) / d ** 0.5
    if spread:
        w = w * (1 + 3 * torch.rand(f, 1, generator=g, device="cuda")) + 0.02
    q = api.exemplar_w4_quantize(w, group)
    return q, torch.as_tensor(ref.w4_load(q.codes.cpu().numpy(), q.words.cpu().numpy(), f, d, group)).cuda()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("n,d", [(1, 1), (3, 31), (16, 128), (19, 300), (33, 129), (70, 1000)])
def test_w4_quantize_and_back(n, d, t, group):
    g = gen("w4", n, d, str(t), group)
    w = (randn(g, n, d) * (0.01 + 3 * torch.rand(n, 1, generator=g, device="cuda"))).to(t)
    w[0, : min(d, 40)] = 0.0
    if n > 2:
        w[1] = w[1].abs() + 1.0
        w[2, d // 2] = float("inf")
    q = api.exemplar_w4_quantize(among_nan(w), group)
    rounded = ref.w4_round(w.float().cpu().numpy(), group)
    codes, words = ref.w4_store(*rounded, group)
    tail = slice(None) if n % 16 == 0 else slice(0, n % 16)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    assert np.array_equal(q.words.cpu().numpy()[:, :, tail], words[:, :, tail])
    values = ref.w4_values(*rounded, group)
    for back in TYPES:
        flat, out = inside((n, d), back, 1)
        got = api.exemplar_w4_dequantize(q, back, out=out)
        want = torch.as_tensor(values).cuda()
        ok = ~want.isnan()
        assert torch.equal(got.isnan(), ~ok) and untouched(flat, 1)
        assert torch.equal(got[ok], want[ok].float().to(back)[()])


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_w4_back_of_many_rows(t):
    """Values past the last-level cache are those of the same rows in small calls (which
    test_w4_quantize_and_back has against its reference)."""
    n, d = glu_sizes.W4_BACK
    q = api.exemplar_w4_quantize(randn(gen("back", str(t)), n, d).to(t), 32)
    flat, out = inside((n, d), t, 1)
    got = api.exemplar_w4_dequantize(q, t, out=out)
    assert untouched(flat, 1)
    for tile in (0, 517, q.codes.shape[0] - 8):
        rows = min(128, n - 16 * tile)
        some = api.W4Rows(q.codes[tile:tile + 8], q.words[tile:tile + 8], rows, d, 32)
        assert torch.equal(got[16 * tile:16 * tile + rows], api.exemplar_w4_dequantize(some, t))


def w4_bounds(x, W, q, bias, t):
    """The sum runs on q and z apart, each up to 15 s |x|: their magnitudes' sum, and
    two more steps for each group."""
    words = torch.as_tensor(q.words.cpu().numpy().view(np.uint32).astype(np.int64)).cuda()
    s = (words & 0xffffff00).to(torch.int32).view(torch.float32).double()  # tiles x groups x 16
    s = s.permute(0, 2, 1).reshape(-1, words.shape[1])[:q.n].repeat_interleave(q.group, 1)[:, :q.d].nan_to_num()
    size = 30 * ref.times(x.abs(), s) + (0 if bias is None else bias.abs())
    length = ((x.shape[1] + 31) // 32 * 8) * (3 if t == torch.float32 else 1) + 2 * (x.shape[1] // q.group + 1) + 16
    e = length * 2.0 ** -23 * size
    y = ref.times(x, W) + (0 if bias is None else bias)
    return y, e, e + ref.half(t) * (y.abs() + e) + ref.TINY[t]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("at,size", list(enumerate(glu_sizes.W4)), ids=str)
def test_w4_product(at, size, t, group):
    n, d, f = size
    g = gen("w4 product", size, str(t), group)
    q, W = weights(g, f, d, group)
    x = randn(g, n, d).to(t)
    bias = randn(g, f) if at % 2 else None
    y, _, bound = w4_bounds(x.double(), W, q, None if bias is None else bias.double(), t)
    flat, out = inside((n, f), t, at % 2)
    got = api.exemplar_w4_product(among_nan(x, at % 2), q, bias=bias, out=out)
    close(got, y, bound)
    assert got is out and untouched(flat, at % 2)
    assert torch.equal(api.exemplar_w4_product(x, q, bias=bias), got)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("at,size", list(enumerate(glu_sizes.W4)), ids=str)
def test_w4_glu(at, size, t, group):
    n, d, f = size
    act, g = ref.ACTIVATIONS[(at + group // 32) % 4], gen("w4 glu", size, str(t), group)
    (qg, Wg), (qu, Wu) = weights(g, f, d, group), weights(g, f, d, group)
    x = randn(g, n, d).to(t)
    bg, bu = (randn(g, f), randn(g, f)) if at % 2 else (None, None)
    flat, out = inside((n, f), t, at % 2)
    got = api.exemplar_w4_glu(among_nan(x, at % 2), qg, qu, bg, bu, activation=ACTS[act], out=out)
    G, eg, _ = w4_bounds(x.double(), Wg, qg, None if bg is None else bg.double(), t)
    U, eu, _ = w4_bounds(x.double(), Wu, qu, None if bu is None else bu.double(), t)
    a, _ = ref.activation(act, G)
    e = 1.2 * eg * (U.abs() + eu) + (a.abs() + ref.act_bound(t) * G.abs()) * eu + ref.act_bound(t) * G.abs() * U.abs()
    close(got, a * U, e + ref.half(t) * ((a * U).abs() + e) + ref.TINY[t])
    assert untouched(flat, at % 2)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", glu_sizes.W4_LARGE, ids=str)
def test_w4_on_many_rows(size, t, group):
    n, d, f = size
    g = gen("w4 many", size, str(t), group)
    (qg, Wg), (qu, Wu) = weights(g, f, d, group), weights(g, f, d, group)
    x, bias = randn(g, n, d).to(t), randn(g, f)
    flat, out = inside((n, f), t, 1)
    api.exemplar_w4_product(among_nan(x), qg, bias=bias, out=out)
    y, _, bound = w4_bounds(x.double(), Wg, qg, bias.double(), t)
    close(out, y, bound)
    assert untouched(flat, 1) and torch.equal(api.exemplar_w4_product(x, qg, bias=bias), out)
    h = api.exemplar_w4_glu(x, qg, qu, bias, None)
    G, eg, _ = w4_bounds(x.double(), Wg, qg, bias.double(), t)
    U, eu, _ = w4_bounds(x.double(), Wu, qu, None, t)
    a, _ = ref.activation("silu", G)
    e = 1.2 * eg * (U.abs() + eu) + (a.abs() + ref.act_bound(t) * G.abs()) * eu + ref.act_bound(t) * G.abs() * U.abs()
    close(h, a * U, e + ref.half(t) * ((a * U).abs() + e) + ref.TINY[t])


@pytest.mark.parametrize("n", [1, 70, 2000])
def test_w4_words_of_any_kind(n):
    """Zero points up to 255, scales of either sign, codes and words of rows past n
    of any kind, and NaN scales."""
    f, d, group = 37, 200, 64
    g = gen("w4 words", n)
    tiles = 3
    codes = torch.randint(0, 256, (tiles, 2, 1024), generator=g, device="cuda").to(torch.uint8)
    s = (0.01 * randn(g, tiles, 4, 16)).view(torch.int32) & -256
    words = s | torch.randint(0, 256, (tiles, 4, 16), generator=g, device="cuda").to(torch.int32)
    words[2, :, 5:] = 0x7fc00000  # past the last row
    words[1, 2, 3] = 0x7fc00000   # row 19
    q = api.W4Rows(codes, words, f, d, group)
    W = torch.as_tensor(ref.w4_load(codes.cpu().numpy(), words.cpu().numpy(), f, d, group)).cuda()
    x = randn(g, n, d)
    got = api.exemplar_w4_product(x, q)
    assert torch.equal(got.isnan(), W.isnan().any(1)[None].expand(n, f))
    ok = ~W.isnan().any(1)
    # 255 + 15 steps of s where w4_bounds has 30
    _, e, _ = w4_bounds(x.double(), W.nan_to_num(), q, None, torch.float32)
    size = 9 * e.abs() + 1e-6
    close(got[:, ok], ref.times(x.double(), W)[:, ok], size[:, ok])


# -- graphs --------------------------------------------------------------------------
def test_captured_and_replayed():
    """Calls without temporary memory in one graph, replayed on new inputs, among
    eager calls; calls with some are refused there and queue nothing."""
    d, f, t = 128, 96, torch.bfloat16
    r = gen("graph")
    x, Wg, Wu, bg, bu = block(r, 4, d, f, t, True)
    many = randn(r, 300, d).to(t)
    q, _ = weights(r, f, d, 64)
    down, _ = weights(r, d, f, 32)
    odd = randn(r, 2000, 333).to(t), randn(r, 2000, 333).to(t)

    def calls():
        h, g, u = api.exemplar_glu(x, Wg, Wu, bg, bu, save=True)
        s = api.exemplar_w4_glu(x, q, q, bg, bu, activation=ACTS["gelu"])
        return [h, g, u, s, api.exemplar_w4_product(s, down), api.exemplar_glu(many, Wg, Wu)[0],
                api.exemplar_w4_product(many, q)]

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
        for bad in (lambda: api.exemplar_glu(odd[0], odd[1], odd[1]),
                    lambda: api.exemplar_glu_backward(out[0], x, Wg, Wu, out[1], out[2])):
            with pytest.raises(api.ExemclError) as e:
                bad()
            assert e.value.status == api.EXEMCL_EINVAL
    for _ in range(4):
        x.copy_(randn(r, 4, d))
        many.copy_(randn(r, 300, d))
        want = calls()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        api.exemplar_glu_backward(want[0], x, Wg, Wu, want[1], want[2])


# -- streams -------------------------------------------------------------------------
def _on_streams():
    import test_streams_gpu as streams
    return streams


@pytest.fixture(scope="module")
def made():
    r = gen("streams")
    n, d, f = 1500, 256, 1000
    x, Wg, Wu, bg, bu = block(r, n, d, f, torch.bfloat16, True)
    q = api.exemplar_w4_quantize(Wg, 64)
    return x, Wg, Wu, bg, bu, randn(r, n, f).bfloat16(), q


CALLS = {
    "glu": (lambda m: m[:5], lambda a, st: api.exemplar_glu(*a, save=True, stream=st)),
    "glu_fp32": (lambda m: tuple(t.float() for t in m[:3]), lambda a, st: api.exemplar_glu(*a, stream=st)[:1]),
    "glu_backward": (lambda m: (m[5], m[0], m[1], m[2], m[5].clone(), m[5].clone()),
                     lambda a, st: api.exemplar_glu_backward(*a, bias=True, stream=st)),
    "w4_quantize": (lambda m: (m[1],), lambda a, st: api.exemplar_w4_quantize(a[0], 32, stream=st)),
    "w4_dequantize": (lambda m: (m[6],), lambda a, st: api.exemplar_w4_dequantize(a[0], torch.float32, stream=st)),
    "w4_product": (lambda m: (m[0], m[6], m[3]), lambda a, st: api.exemplar_w4_product(*a, stream=st)),
    "w4_glu": (lambda m: (m[0], m[6], m[6], m[3], m[4]), lambda a, st: api.exemplar_w4_glu(*a, stream=st)),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream(name, made, monkeypatch):
    """As the other calls do it: whose memory results are, and when memory that is
    freed early is used again."""
    streams = _on_streams()
    monkeypatch.setattr(streams, "CALLS", CALLS)

    def copies(a):
        return tuple(x._replace(codes=x.codes.clone(), words=x.words.clone()) if isinstance(x, api.W4Rows) else x.clone()
                     for x in a)

    monkeypatch.setattr(streams, "copies", copies)
    streams.test_memory_of_a_call_on_another_stream(name, made)


def test_calls_from_several_threads():
    """Threads that share a stream, and threads with streams of their own, get the
    results of calls made one after the other."""
    import threading
    r = gen("threads")
    n, d, f, t = 200, 136, 150, torch.float32
    sets = [block(gen("threads", i), n, d, f, t, False)[:3] for i in range(4)]
    dh = randn(r, n, f)
    want = []
    for x, Wg, Wu in sets:
        h, g, u = api.exemplar_glu(x, Wg, Wu, save=True)
        want.append([h, *api.exemplar_glu_backward(dh, x, Wg, Wu, g, u)[:3]])
    torch.cuda.synchronize()
    got = [None] * 8

    def work(i):
        x, Wg, Wu = sets[i % 4]
        st = torch.cuda.Stream() if i >= 4 else None
        with torch.cuda.stream(st or torch.cuda.current_stream()):
            for _ in range(5):
                h, g, u = api.exemplar_glu(x, Wg, Wu, save=True)
                out = [h, *api.exemplar_glu_backward(dh, x, Wg, Wu, g, u)[:3]]
        torch.cuda.synchronize()
        got[i] = out

    threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    for i in range(8):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i % 4])), i


def test_gradient_within_a_workspace_limit(monkeypatch):
    """Without memory for partial sums the products are not divided; without memory
    for the rest the call is refused."""
    n, d, f, t = 4000, 64, 72, torch.bfloat16
    r = gen("limit")
    x, Wg, Wu, _, _ = block(r, n, d, f, t, False)
    dh, g, u = (randn(r, n, f).to(t) for _ in range(3))
    args = (dh, x, Wg, Wu, g, u)
    want, bounds = ref.glu_backward(*wide(*args), "silu"), ref.backward_bounds(*wide(*args), "silu", t)
    own = 2 * n * f * 2
    for limit in (None, own + 4096, own - 4096):
        if limit:
            monkeypatch.setenv("EXEMCL_WORKSPACE_LIMIT", str(limit))
        if limit and limit < own:
            with pytest.raises(api.ExemclError) as e:
                api.exemplar_glu_backward(*args)
            assert e.value.status == api.EXEMCL_ENOMEM
            continue
        for a, w, b in zip(api.exemplar_glu_backward(*args)[:3], want, bounds):
            close(a, w, b)


# -- together -----------------------------------------------------------------------
def test_norm_block_and_products_together():
    """A residual block as it is trained and served: norm, gated block, the product
    behind it, and back; then the block and the product on 4-bit weights.  Each
    against its 64-bit form on the step's own input."""
    n, d, f, t = 300, 192, 320, torch.bfloat16
    r = gen("together")
    stream, res = randn(r, n, d).to(t), randn(r, n, d).to(t)
    w = (1 + 0.1 * randn(r, d)).to(t)
    _, Wg, Wu, _, _ = block(r, n, d, f, t, False)
    y, h, rstd = api.exemplar_rmsnorm(stream, w, res)
    act, g, u = api.exemplar_glu(y, Wg, Wu, save=True)
    for got, want, b in zip((act, g, u), ref.glu(*wide(y, Wg, Wu, None, None), "silu"),
                            ref.glu_bounds(*wide(y, Wg, Wu, None, None), "silu", t)):
        close(got, want, b)
    dh = randn(r, n, f).to(t)
    args = (dh, y, Wg, Wu, g, u)
    dy, dWg, dWu, _, _ = api.exemplar_glu_backward(*args)
    for got, want, b in zip((dy, dWg, dWu), ref.glu_backward(*wide(*args), "silu"), ref.backward_bounds(*wide(*args), "silu", t)):
        close(got, want, b)
    dx, dw = api.exemplar_rmsnorm_backward(dy, h, w, rstd)
    assert bool(dx.isfinite().all()) and bool(dw.isfinite().all())
    qg, qu = api.exemplar_w4_quantize(Wg, 32), api.exemplar_w4_quantize(Wu, 32)
    down, D = weights(r, d, f, 64)
    for rows in (1, n):
        s = api.exemplar_w4_glu(y[:rows], qg, qu)
        out = api.exemplar_w4_product(s, down)
        want, _, bound = w4_bounds(s.double(), D, down, None, t)
        close(out, want, bound)
        # 4-bit weights: a step of a sixteenth of the range is 1/3 of a weight's
        # size, half of it at most, 1/10 on average, and so for both factors of h
        assert float((s.double() - act[:rows].double()).square().mean() / act[:rows].double().square().mean()) < 0.15 ** 2 * 2


def example():
    spec = importlib.util.spec_from_file_location(
        "gated_block", pathlib.Path(__file__).parent.parent / "examples" / "gated_block.py")
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_runs():
    losses, off, f = example().main(["--n", "700", "--width", "192", "--inner", "320", "--steps", "3"])
    assert len(losses) == 3 and all(np.isfinite(losses)) and np.isfinite(off) and bool(f.isfinite().all())


def test_example_gradients():
    """The example's gradients against PyTorch's of the whole block in 64 bits.  Off by
    roundings to bf16 (half a step 2^-9): of y, of g and u, of dh, of dg, of the result,
    of h in no gradient; each moves a term of the sums by chance, so the root mean
    square of all is within sqrt(5) 2^-9 and a factor of 2 for slopes above 1."""
    ex, (n, d, f) = example(), (300, 96, 160)
    r = gen("example")
    x = randn(r, n, d).bfloat16()
    Wg, Wu = ((randn(r, f, d) / d ** 0.5).bfloat16() for _ in range(2))
    Wd = (randn(r, d, f) / f ** 0.5).bfloat16()
    dz = randn(r, n, d)
    _, kept = ex.forward(x, Wg, Wu, Wd)
    got = ex.gradients(dz, kept, Wg, Wu, Wd)
    leaves = [Wg.double().requires_grad_(), Wu.double().requires_grad_()]
    x64 = x.double()
    y = x64 / torch.sqrt((x64 * x64).mean(1, keepdim=True) + ex.EPS)
    z = x64 + (torch.nn.functional.silu(y @ leaves[0].t()) * (y @ leaves[1].t())) @ Wd.double().t()
    z.backward(dz.double())
    for a, w in zip(got, leaves):
        off = float((a.double() - w.grad).square().mean().sqrt() / w.grad.square().mean().sqrt())
        assert off < 2 * 5 ** 0.5 * 2.0 ** -9, off
