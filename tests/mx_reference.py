"""Plain 64-bit forms (numpy, on the host) of the operators on microscaled
rows, for the tests."""
import numpy as np

FP4, FP8 = 4, 8


def table(fmt):
    """The non-negative values of an element type, in code order."""
    if fmt == FP4:
        return np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


def padded(d):
    return (d + 127) // 128 * 128


def element_codes(v, fmt):
    """Nearest codes, ties to the even one, magnitudes past the largest at it."""
    t = table(fmt)
    a = np.minimum(np.abs(v), t[-1])
    hi = np.searchsorted(t, a).clip(max=len(t) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = t[hi] - a, a - t[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(t[hi] == a, hi, code)
    return code + np.where(np.signbit(v), 8 if fmt == FP4 else 128, 0)


def quantize(x, fmt):
    """(codes, scales) of x (float64, n x d), padded as they are stored."""
    n, d = x.shape
    dp = padded(d)
    y = np.zeros((n, dp))
    y[:, :d] = x
    y = y.reshape(n, dp // 32, 32)
    big = np.abs(y).max(2)
    fine = np.isfinite(big)
    _, e = np.frexp(np.where(fine, big, 1.0))
    scale = np.where(big > 0, np.clip(e - 1 - (2 if fmt == FP4 else 8), -127, 127) + 127, 0)
    with np.errstate(all="ignore"):
        v = np.ldexp(y, -(scale - 127)[:, :, None])
    codes = element_codes(np.where(fine[:, :, None], v, 0.0), fmt).reshape(n, dp)
    scale = np.where(fine, scale, 255).astype(np.uint8)
    if fmt == FP4:
        codes = codes[:, 0::2] + 16 * codes[:, 1::2]
    return codes.astype(np.uint8), scale


def values(codes, scales, d, fmt):
    """What stored rows stand for, float64 n x d."""
    codes, scales = np.asarray(codes).astype(np.int64), np.asarray(scales).astype(np.int64)
    t = table(fmt)
    if fmt == FP4:
        t = np.concatenate([t, -t])
        codes = np.stack([codes & 15, codes >> 4], 2).reshape(len(codes), -1)
    else:
        t = np.concatenate([t, [np.nan], -t, [np.nan]])
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales - 127))
    return (t[codes] * np.repeat(f, 32, 1))[:, :d]


def rmsnorm(x, w, r, eps):
    """(y, v, rstd)."""
    v = x if r is None else x + r
    rstd = 1.0 / np.sqrt((v * v).mean(1) + eps)
    return v * rstd[:, None] * (1.0 if w is None else w), v, rstd


def rmsnorm_backward(dy, h, w, rstd, dh):
    """(dx, dw)."""
    xhat = h * rstd[:, None]
    g = dy if w is None else dy * w
    dx = rstd[:, None] * (g - xhat * (g * xhat).mean(1, keepdims=True))
    return dx if dh is None else dx + dh, (dy * xhat).sum(0)


def f_of_sets(V, sets):
    """f(S) of every set (index lists without empty slots), directly from Eq. (3)
    and Eq. (4): squared distances, the zero vector a member of every set."""
    e0 = (V * V).sum(1)
    out = []
    for s in sets:
        near = e0.copy()
        for i in s:
            near = np.minimum(near, ((V - V[i]) ** 2).sum(1))
        out.append(e0.mean() - near.mean())
    return np.array(out)
