"""The gated feed-forward operators: both projections, the activation and their
product in one call, their gradient, and the same on 4-bit weights with group
scales.

Between the norm that ends the residual stream's addition and the projection that
makes an embedding stands a gated block, h = act(x Wg' + bg) * (x Wu' + bu).  It
is trained with weights of the rows' type and served with weights of 4 bits, one
scale and zero point for 32, 64 or 128 of them, where a product by such weights is
also what follows it.

``listed()`` names the timed cases, ``draw()`` makes more of the same ranges,
``prepare()`` builds the inputs on the GPU from a seed, ``run()`` is one call:
elementary torch operations in 32 bits where ``own`` is false, the library's
operators where it is true.  ``work()`` says what a call cannot do without, and
``exact()`` is the same result from the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
ACTIVATIONS = ("silu", "gelu", "gelu_tanh", "relu")
TILE, ROW = 16, 128   # stored 4-bit weights: tiles of 16 rows x 128 coordinates


# -- cases -------------------------------------------------------------------
def _glu(n, d, f, dtype, act="silu", bias=False, save=False):
    return {"op": "glu", "n": n, "d": d, "f": f, "dtype": dtype, "act": act, "bias": bias, "save": save}


def _grad(n, d, f, dtype, act="silu", bias=False):
    return {"op": "grad", "n": n, "d": d, "f": f, "dtype": dtype, "act": act, "bias": bias}


def _w4(n, d, f, dtype, group=128, bias=False):
    return {"op": "w4", "n": n, "d": d, "f": f, "dtype": dtype, "group": group, "bias": bias}


def _w4_glu(n, d, f, dtype, group=128, act="silu", bias=False):
    return {"op": "w4_glu", "n": n, "d": d, "f": f, "dtype": dtype, "group": group, "act": act, "bias": bias}


def listed():
    cases = {
        # One row while serving with unrounded weights: every weight is read once.
        "glu_one_row": _glu(1, 1536, 4096, "bf16"),
        # A short batch in fp32 where nothing is a multiple of anything, kept for
        # the gradient.
        "glu_ragged_fp32": _glu(333, 301, 1111, "fp32", "gelu", bias=True, save=True),
        # The forward half of a training step on many rows, kept for the gradient.
        "glu_large_bf16": _glu(16_384, 4096, 8192, "bf16", save=True),
        # The gradient of a short ragged batch in fp16.
        "grad_ragged_fp16": _grad(517, 301, 777, "fp16", "gelu_tanh", bias=True),
        # The backward half of a training step at an embedding model's width.
        "grad_step_bf16": _grad(8192, 1536, 4096, "bf16"),
        # The same for a wide model's.
        "grad_large_bf16": _grad(16_384, 4096, 8192, "bf16"),
        # One row through the product behind the block, 4-bit weights.
        "w4_one_row": _w4(1, 8192, 4096, "bf16"),
        # A few rows, odd sizes, groups of 64, with a bias.
        "w4_ragged_fp16": _w4(7, 1001, 1537, "fp16", 64, bias=True),
        # A long text's rows at once by the same kind of weights.
        "w4_rows_bf16": _w4(2048, 4096, 8192, "bf16"),
        # One row through the block on 4-bit weights.
        "w4_glu_one_row": _w4_glu(1, 4096, 8192, "bf16"),
        # A serving batch: a row for each of its requests, groups of 32.
        "w4_glu_batch_fp16": _w4_glu(24, 1536, 4096, "fp16", 32, "gelu_tanh", bias=True),
        # Requests' whole texts in one batch.
        "w4_glu_rows_bf16": _w4_glu(1000, 1536, 4096, "bf16", 64),
    }
    return [{"name": name, **c} for name, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of the sizes are whole multiples of 64."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.5 else max(64, v // 64 * 64)


def draw(rng):
    op = rng.choices(["glu", "grad", "w4", "w4_glu"], [4, 3, 4, 4])[0]
    dtype = rng.choice(["fp32", "fp16", "bf16", "bf16"])
    act, bias = rng.choice(ACTIVATIONS), rng.random() < 0.5
    d, f = _size(rng, 32, 4096), _size(rng, 32, 8192)
    if op in ("glu", "grad"):
        n = _log(rng, 1, 16_384)
        if dtype == "fp32":
            n = max(1, min(n, 90_000_000_000 // (d * f)))
        return _grad(n, d, f, dtype, act, bias) if op == "grad" else _glu(n, d, f, dtype, act, bias, rng.random() < 0.5)
    group = rng.choice([32, 64, 128])
    n = _log(rng, 1, 16) if rng.random() < 0.5 else _log(rng, 1, 2048)
    if dtype == "fp32":
        n = min(n, 512)
    if op == "w4":
        return _w4(n, f, d, dtype, group, bias) if rng.random() < 0.5 else _w4(n, d, f, dtype, group, bias)
    return _w4_glu(n, d, f, dtype, group, act, bias)


# -- 4-bit weights as the library stores them -----------------------------------
def _round_weights(w, group):
    """(codes 0..15, scales, zero points) of w: value = (code - zero) * scale."""
    n, d = w.shape
    groups = (d + group - 1) // group
    v = torch.nn.functional.pad(w, (0, groups * group - d)).view(n, groups, group)
    lo, hi = v.amin(2).clamp(max=0.0), v.amax(2).clamp(min=0.0)
    s = (hi - lo) / 15.0
    s = ((s.view(torch.int32) + 255) & -256).view(torch.float32)  # 16 significant bits, upwards
    inv = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    zero = torch.round(-lo * inv).clamp(0, 15)
    q = (torch.round(v * inv[:, :, None]) + zero[:, :, None]).clamp(0, 15)
    return q.flatten(1)[:, :d].to(torch.uint8), s, zero.to(torch.int32)


def _stored(w, group):
    """(codes, words): tiles of 16 rows x 128 coordinates, in them 16 bytes for each
    row and quarter, whose dword j holds coordinates 32 j + 8 quarter + 0..7 (the
    first four in the low halves of its bytes); a word for each group, the scale with
    its zero point in the last 8 bits."""
    q, s, zero = _round_weights(w, group)
    n, d = q.shape
    tiles, blocks = (n + TILE - 1) // TILE, (d + ROW - 1) // ROW
    full = torch.zeros(tiles * TILE, blocks * ROW, dtype=torch.uint8, device=q.device)
    full[:n, :d] = q
    # (tile, row, block, dword, quarter, half, byte) -> (tile, block, quarter, row, dword, byte)
    v = full.view(tiles, TILE, blocks, 4, 4, 2, 4)
    codes = (v[:, :, :, :, :, 0] + 16 * v[:, :, :, :, :, 1]).permute(0, 2, 4, 1, 3, 5)
    words = torch.zeros(tiles * TILE, blocks * ROW // group, dtype=torch.int32, device=q.device)
    words[:n, :s.shape[1]] = s.view(torch.int32) + zero
    words = words.view(tiles, TILE, -1).permute(0, 2, 1)
    return codes.reshape(tiles, blocks, TILE * ROW // 2).contiguous(), words.contiguous()


def _loaded(stored, n, d, group):
    """The values of stored weights, in fp32."""
    codes, words = stored
    tiles, blocks = codes.shape[:2]
    v = codes.view(tiles, blocks, 4, TILE, 4, 4)
    q = torch.stack((v & 15, v >> 4), 5).permute(0, 3, 1, 4, 2, 5, 6).reshape(tiles * TILE, -1, group).float()
    w = words.permute(0, 2, 1).reshape(tiles * TILE, -1)
    s, zero = (w & -256).view(torch.float32), (w & 255).float()
    return ((q - zero[:, :, None]) * s[:, :, None]).flatten(1)[:n, :d]


# -- inputs --------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def prepare(case, seed):
    c, g = case, _generator(seed)
    n, d, f, T = c["n"], c["d"], c["f"], DTYPES[c["dtype"]]
    s = {"c": dict(case), "x": _randn(g, n, d).to(T)}
    names = ("W",) if c["op"] == "w4" else ("Wg", "Wu")
    for name in names:
        w = _randn(g, f, d) / math.sqrt(d)
        s[name] = _stored(w, c["group"]) if c["op"].startswith("w4") else w.to(T)
        s["b" + name[1:]] = 0.1 * _randn(g, f) if c["bias"] else None
    if c["op"] == "grad":
        s["dh"] = (0.1 * _randn(g, n, f)).to(T)
        for name in ("g", "u"):
            p = s["x"].float() @ s["W" + name].float().t()
            s[name] = (p if s["b" + name] is None else p + s["b" + name]).to(T)
    return s


# -- one pass --------------------------------------------------------------------
def _activation(name, g):
    if name == "silu":
        return g / (1.0 + torch.exp(-g))
    if name == "gelu":
        return 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))
    return g.clamp(min=0.0)


def _slope(name, g):
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return p * (1.0 + g * (1.0 - p))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        a = math.sqrt(2.0 / math.pi)
        t = torch.tanh(a * (g + 0.044715 * g * g * g))
        return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * a * (1.0 + 3.0 * 0.044715 * g * g)
    return (g > 0).to(g.dtype)


def _project(x, w, b):
    p = x @ w.t()
    return p if b is None else p + b


def _plain(s):
    c = s["c"]
    T, x = DTYPES[c["dtype"]], s["x"].float()
    if c["op"] == "w4":
        return _project(x, _loaded(s["W"], c["f"], c["d"], c["group"]), s["b"]).to(T)
    if c["op"] == "grad":
        g, u, dh = s["g"].float(), s["u"].float(), s["dh"].float()
        dg, du = dh * u * _slope(c["act"], g), dh * _activation(c["act"], g)
        out = [(dg @ s["Wg"].float() + du @ s["Wu"].float()).to(T), (dg.t() @ x).to(T), (du.t() @ x).to(T)]
        return out + [dg.sum(0), du.sum(0)] if c["bias"] else out
    if c["op"] == "w4_glu":
        Wg, Wu = (_loaded(s[w], c["f"], c["d"], c["group"]) for w in ("Wg", "Wu"))
    else:
        Wg, Wu = s["Wg"].float(), s["Wu"].float()
    g, u = _project(x, Wg, s["bg"]), _project(x, Wu, s["bu"])
    h = (_activation(c["act"], g) * u).to(T)
    return [h, g.to(T), u.to(T)] if c.get("save") else h


def _own(s):
    from paper_2101_08763_amd import api

    c = s["c"]
    f, d, group = c["f"], c["d"], c.get("group")
    if c["op"] == "w4":
        return api.exemplar_w4_product(s["x"], api.W4Rows(*s["W"], f, d, group), bias=s["b"])
    act = {"silu": api.EXEMCL_SILU, "gelu": api.EXEMCL_GELU, "gelu_tanh": api.EXEMCL_GELU_TANH,
           "relu": api.EXEMCL_RELU}[c["act"]]
    if c["op"] == "w4_glu":
        return api.exemplar_w4_glu(s["x"], api.W4Rows(*s["Wg"], f, d, group), api.W4Rows(*s["Wu"], f, d, group),
                                   s["bg"], s["bu"], activation=act)
    if c["op"] == "grad":
        out = api.exemplar_glu_backward(s["dh"], s["x"], s["Wg"], s["Wu"], s["g"], s["u"], activation=act, bias=c["bias"])
        return list(out) if c["bias"] else list(out[:3])
    h, g, u = api.exemplar_glu(s["x"], s["Wg"], s["Wu"], s["bg"], s["bu"], activation=act, save=c["save"])
    return [h, g, u] if c["save"] else h


def run(state):
    return _own(state) if own else _plain(state)


# -- what a pass cannot do without -------------------------------------------------
def work(case):
    c = case
    n, d, f, es = c["n"], c["d"], c["f"], BYTES[c["dtype"]]
    if c["op"] == "grad":
        moved = (3 * n * f + 2 * n * d + 4 * f * d) * es + (8 * f if c["bias"] else 0)
        return {"bytes": moved, "flops": 8.0 * n * d * f}
    both = 1 if c["op"] == "w4" else 2
    if c["op"] == "glu":
        weights = f * d * es
    else:
        weights = f * (d / 2 + 4 * ((d + c["group"] - 1) // c["group"]))
    out = 3 if c.get("save") else 1
    moved = n * d * es + both * (weights + (4 * f if c["bias"] else 0)) + out * n * f * es
    return {"bytes": moved, "flops": 2.0 * both * n * d * f}


# -- the definition in 64 bits -------------------------------------------------------
def _exact_weights(stored, n, d, group):
    """(code - zero) * scale, by the place of every coordinate."""
    codes, words = stored
    k = torch.arange(d, device="cuda")
    byte = (k % 32 // 8) * 256 + (k % 128 // 32) * 4 + k % 4       # of row 0 in its tile
    i = torch.arange(n, device="cuda")[:, None]
    at = codes[i // TILE, (k // ROW)[None], byte[None] + 16 * (i % TILE)].long()
    q = torch.where((k % 8 >= 4)[None], at // 16, at % 16).double()
    word = words[i // TILE, (k // group)[None], i % TILE]
    zero = word & 255
    return (q - zero.double()) * (word - zero).view(torch.float32).double()


def _exact_pair(name, g):
    """The activation and its derivative at g."""
    if name == "relu":
        on = (g > 0).double()
        return g * on, on
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1.0 - p)
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * cdf, cdf + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
    # (1 + tanh z) / 2 = sigmoid(2 z)
    z = math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)
    p = torch.sigmoid(z)
    return g * p, p + g * p * (1.0 - p) * math.sqrt(8.0 / math.pi) * (1.0 + 3.0 * 0.044715 * g ** 2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    n, d, f = c["n"], c["d"], c["f"]
    x = s["x"].double()

    def through(name):
        w = _exact_weights(s["W" + name], f, d, c["group"]) if "group" in c else s["W" + name].double()
        y = x @ w.t().contiguous()
        return y if s["b" + name] is None else y + s["b" + name].double()

    if c["op"] == "w4":
        return through("")
    if c["op"] == "grad":
        dh, u = s["dh"].double(), s["u"].double()
        a, slope = _exact_pair(c["act"], s["g"].double())
        dg, du = slope * u * dh, a * dh
        dx = torch.cat((dg, du), 1) @ torch.cat((s["Wg"], s["Wu"])).double()
        out = [dx, dg.t().contiguous() @ x, du.t().contiguous() @ x]
        return out + [dg.sum(0), du.sum(0)] if c["bias"] else out
    g, u = through("g"), through("u")
    h = _exact_pair(c["act"], g)[0] * u
    return [h, g, u] if c.get("save") else h
