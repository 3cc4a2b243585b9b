"""Plain 64-bit forms (torch, on whatever device the tensors are) of the gated
feed-forward block, its gradient and weights of 4 bits with group scales, with the
bounds the tests hold results to."""
import math

import numpy as np
import torch

ACTIVATIONS = ("silu", "gelu", "gelu_tanh", "relu")  # in the order of exemcl_activation


def activation(name, g):
    """(a(g), a'(g)) in float64."""
    if name == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    if name == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    # (1 + tanh z) / 2 = sigmoid(2 z), which keeps its digits where tanh z is near -1
    z2 = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
    s = torch.sigmoid(z2)
    return g * s, s + g * s * torch.sigmoid(-z2) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g * g)


def times(a, b):
    """a b' in float64."""
    return a @ b.t().contiguous()


def glu(x, Wg, Wu, bg, bu, act):
    g, u = times(x, Wg), times(x, Wu)
    g, u = (g if bg is None else g + bg), (u if bu is None else u + bu)
    return activation(act, g)[0] * u, g, u


def glu_backward(dh, x, Wg, Wu, g, u, act):
    a, slope = activation(act, g)
    dg, du = dh * u * slope, dh * a
    return dg @ Wg + du @ Wu, times(dg.t().contiguous(), x.t()), times(du.t().contiguous(), x.t()), dg.sum(0), du.sum(0)


# -- bounds -----------------------------------------------------------------------
# A result of type T is off by half a step, eps(T) / 2 of it (and half the smallest
# subnormal), beside what its fp32 sum is off by.  A sum of n products: each
# instruction adds 32 of them in at most 8 steps, wavefronts' and parts' sums take
# 16 more at most, six products of fp32's parts six times as many, and a step is off
# by at most one unit of 2^-23 of the sum of magnitudes (truncation allowed); what
# fp32's parts leave out is 2^-25 of it.
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}


def half(t):
    return torch.finfo(t).eps / 2


def steps(n, t):
    return ((n + 31) // 32 * 8) * (6 if t == torch.float32 else 1) + 16


def sum_bound(n, t):
    return steps(n, t) * 2.0 ** -23 + (2.0 ** -25 if t == torch.float32 else 0.0)


# Of an activation or its derivative: the instructions' exponential and reciprocal
# (16-bit types) or the library's (fp32), relative to their largest factors.
def act_bound(t):
    return 2.0 ** -20 if t == torch.float32 else 2.0 ** -18


def project_bounds(x, W, b, t):
    size = times(x.abs(), W.abs())
    return sum_bound(x.shape[1], t) * (size if b is None else size + b.abs())


def glu_bounds(x, Wg, Wu, bg, bu, act, t):
    """Bounds of (h, g, u)."""
    _, g, u = glu(x, Wg, Wu, bg, bu, act)
    eg, eu = project_bounds(x, Wg, bg, t), project_bounds(x, Wu, bu, t)
    a, _ = activation(act, g)
    # |a'| <= 1.13
    before = 1.2 * eg * (u.abs() + eu) + (a.abs() + act_bound(t) * g.abs()) * eu + act_bound(t) * g.abs() * u.abs()
    rounded = [(before, a * u), (eg, g), (eu, u)]
    return [e + half(t) * (v.abs() + e) + TINY[t] for e, v in rounded]


def backward_bounds(dh, x, Wg, Wu, g, u, act, t):
    """Bounds of (dx, dWg, dWu, dbg, dbu)."""
    a, slope = activation(act, g)
    dg, du = dh * u * slope, dh * a
    # dg and du before they are rounded, and after
    eg, eu = act_bound(t) * (dh * u).abs() * (1 + g.abs()), act_bound(t) * (dh * g).abs()
    rounding = 2.0 ** -25 if t == torch.float32 else half(t)
    rg, ru = eg + rounding * (dg.abs() + eg) + TINY[t], eu + rounding * (du.abs() + eu) + TINY[t]
    n, f = dh.shape
    out = []
    for err, size, value, length in (
            (rg @ Wg.abs() + ru @ Wu.abs(), dg.abs() @ Wg.abs() + du.abs() @ Wu.abs(), dg @ Wg + du @ Wu, 2 * f),
            (times(rg.t().contiguous(), x.abs().t()), times(dg.abs().t().contiguous(), x.abs().t()), times(dg.t().contiguous(), x.t()), n),
            (times(ru.t().contiguous(), x.abs().t()), times(du.abs().t().contiguous(), x.abs().t()), times(du.t().contiguous(), x.t()), n)):
        e = err + sum_bound(length, t) * size
        out.append(e + half(t) * (value.abs() + e) + TINY[t])
    for err, v in ((eg, dg), (eu, du)):
        # a thread's rows in turn, 8 threads, then 64 bits; rounded once
        out.append(err.sum(0) + (-(-n // 8) + 9) * 2.0 ** -24 * v.abs().sum(0) + 2.0 ** -24 * v.sum(0).abs() + 2.0 ** -126)
    return out


# -- 4-bit weights, numpy ------------------------------------------------------------
def w4_round(w, group):
    """(q, s, z) of w (float32, n x d) by the rule of exemcl.h: q n x d, s and z n x
    groups, step by step in the precision that it names."""
    n, d = w.shape
    groups = -(-d // group)
    v = np.zeros((n, groups * group), np.float32)
    v[:, :d] = w
    v = v.reshape(n, groups, group)
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[:, :, None], np.float32(0), v)
    lo, hi = np.minimum(v.min(2), 0), np.maximum(v.max(2), 0)
    s0 = (hi * np.float32(0.5) - lo * np.float32(0.5)) / np.float32(7.5)
    s = ((s0.view(np.uint32) + np.uint32(255)) & np.uint32(0xffffff00)).view(np.float32)
    s = np.where(s0 < np.float32(2.0 ** -126), np.float32(0), s)
    with np.errstate(divide="ignore"):
        r = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
    z = np.clip(np.rint(-lo * r), 0, 15)
    q = np.clip(np.rint(v * r[:, :, None]) + z[:, :, None], 0, 15)
    s = np.where(bad, np.float32(np.nan), s)
    return np.where(bad[:, :, None], 0, q).reshape(n, -1)[:, :d].astype(np.int64), s, np.where(bad, 0, z).astype(np.int64)


def w4_values(q, s, z, group):
    d = q.shape[1]
    return (q - np.repeat(z, group, 1)[:, :d]) * np.repeat(s.astype(np.float64), group, 1)[:, :d]


def w4_store(q, s, z, group):
    """(codes, words) by exemcl.h's formula for each coordinate's place."""
    n, d = q.shape
    tiles, blocks = -(-n // 16), -(-d // 128)
    codes = np.zeros((tiles, blocks, 1024), np.uint8)
    for i in range(n):
        for k in range(d):
            j, p, e = k % 128 // 32, k % 32 // 8, k % 8
            codes[i // 16, k // 128, 256 * p + 16 * (i % 16) + 4 * j + e % 4] |= q[i, k] << (4 if e >= 4 else 0)
    words = np.zeros((tiles, blocks * 128 // group, 16), np.uint32)
    bits = np.where(np.isnan(s), np.uint32(0x7fc00000), s.astype(np.float32).view(np.uint32))
    for i in range(n):
        words[i // 16, :s.shape[1], i % 16] = bits[i] | z[i].astype(np.uint32)
    return codes, words.view(np.int32)


def w4_load(codes, words, n, d, group):
    """The values (float64) of stored weights, n x d."""
    i, k = np.arange(n)[:, None], np.arange(d)[None]
    byte = codes[i // 16, k // 128, 256 * (k % 32 // 8) + 16 * (i % 16) + 4 * (k % 128 // 32) + k % 4]
    q = np.where(k % 8 >= 4, byte >> 4, byte & 15).astype(np.float64)
    w = words.view(np.uint32)[i // 16, k // group, i % 16]
    s = (w & np.uint32(0xffffff00)).view(np.float32).astype(np.float64)
    return (q - (w & np.uint32(255))) * s
