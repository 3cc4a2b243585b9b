"""Choosing exemplars among embeddings that are made and kept in 4 and 8 bits.

    python examples/select_embeddings.py [--n 20000 --hidden 1024 --dim 512]

Hidden states and their residual stream are normalised to 8-bit rows, projected
by 4-bit weights, and the embeddings kept as 4-bit rows, on which candidate sets
are scored; the best ones are scored again on the unrounded embeddings.  Before
that the norm's weight is trained for a few steps, so that the projection by
rounded weights comes near the one by the weights they were made from.
"""
from __future__ import annotations

import argparse
import pathlib
import sys

import torch

sys.path.insert(0, str(pathlib.Path(__file__).resolve().parent.parent))
from paper_2101_08763_amd import api  # noqa: E402

FP4, FP8 = api.EXEMCL_MXFP4, api.EXEMCL_MXFP8
EPS = 1e-5


def train(x, r, weight, W, target, steps, rate):
    """Steps of gradient descent on mean ||E - target||^2 by the norm's weight;
    the loss before each."""
    losses = []
    back = api.exemplar_mx_dequantize(W, torch.float32)  # dE W, for the norm's gradient
    for _ in range(steps):
        w = weight.to(x.dtype)
        y, h, rstd = api.exemplar_rmsnorm(x, w, r, eps=EPS, format=FP8)
        diff = api.exemplar_mx_product(y, W) - target
        losses.append(float(diff.square().mean()))
        dy = ((2.0 / diff.numel()) * (diff @ back)).to(x.dtype)
        _, dw = api.exemplar_rmsnorm_backward(dy, h, w, rstd)
        weight -= rate * dw
    return losses


def embed(x, r, weight, W):
    """4-bit embeddings, and the bf16 ones they are rounded from."""
    y, _, _ = api.exemplar_rmsnorm(x, weight.to(x.dtype), r, eps=EPS, format=FP8)
    E = api.exemplar_mx_product(y, W, dtype=torch.bfloat16)
    return api.exemplar_mx_quantize(E, FP4), E


def select(q, E, sets, best=16):
    """The sets with the highest f on the 4-bit rows, f there and on E."""
    f = api.exemplar_mx_eval(q, sets)
    at = f.topk(min(best, f.numel())).indices
    return at, f[at], api.exemplar_eval(E, sets[at].contiguous())


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--n", type=int, default=20_000, help="rows")
    p.add_argument("--hidden", type=int, default=1024, help="width of the hidden states")
    p.add_argument("--dim", type=int, default=512, help="width of the embeddings")
    p.add_argument("--sets", type=int, default=512)
    p.add_argument("--members", type=int, default=16)
    p.add_argument("--steps", type=int, default=5)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    topics = 3.0 * randn(20, a.hidden)
    x = (randn(a.n, a.hidden) + topics[torch.randint(0, 20, (a.n,), generator=g, device="cuda")]).bfloat16()
    r = randn(a.n, a.hidden).bfloat16()
    full = randn(a.dim, a.hidden) / a.hidden ** 0.5
    W = api.exemplar_mx_quantize(full, FP4)
    v = x.float() + r.float()
    target = (v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)) @ full.t()
    weight = torch.ones(a.hidden, device="cuda")
    losses = train(x, r, weight, W, target, a.steps, rate=0.2 * a.dim)
    print("mean squared distance to the unrounded projection: " + " ".join("%.5f" % t for t in losses))

    q, E = embed(x, r, weight, W)
    bits = (q.codes.numel() + q.scales.numel()) * 8 / E.numel()
    print("embeddings: %d x %d in %.2f bits an element" % (*E.shape, bits))
    sets = torch.randint(0, a.n, (a.sets, a.members), generator=g, device="cuda", dtype=torch.int32)
    at, f4, f = select(q, E, sets)
    for j, u, w in zip(at[:5].tolist(), f4.tolist(), f.tolist()):
        print("set %4d: f %.4f on 4-bit rows, %.4f on bf16 rows" % (j, u, w))
    return losses, f4, f


if __name__ == "__main__":
    main()
