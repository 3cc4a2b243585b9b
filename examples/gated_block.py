"""A gated residual block before the embeddings: trained in bf16, served in 4 bits.

    python examples/gated_block.py [--n 4096 --width 512 --inner 1024]

The block is z = x + h Wd', h = silu(y Wg') * (y Wu') with y the norm of x.  Its gated
weights are trained for a few steps towards another block's z; then all three weights
are rounded to 4 bits with a scale for 64 of them, the block runs on those, and its
results are normalised to 4-bit rows on which sets of exemplars are chosen.
"""
from __future__ import annotations

import argparse
import pathlib
import sys

import torch

sys.path.insert(0, str(pathlib.Path(__file__).resolve().parent.parent))
from paper_2101_08763_amd import api  # noqa: E402

EPS = 1e-5


def forward(x, Wg, Wu, Wd):
    """z in fp32, and what the gradient needs."""
    y, _, _ = api.exemplar_rmsnorm(x, eps=EPS)
    h, g, u = api.exemplar_glu(y, Wg, Wu, save=True)
    return x.float() + h.float() @ Wd.float().t(), (y, g, u)


def gradients(dz, kept, Wg, Wu, Wd):
    """dWg and dWu from dz (fp32)."""
    y, g, u = kept
    dh = (dz @ Wd.float()).to(y.dtype)
    _, dWg, dWu, _, _ = api.exemplar_glu_backward(dh, y, Wg, Wu, g, u)
    return dWg, dWu


def train(x, target, Wg, Wu, Wd, steps, rate):
    """Steps of gradient descent on mean ||z - target||^2 by Wg and Wu (kept in fp32);
    the loss before each."""
    losses, master = [], [Wg.float(), Wu.float()]
    for _ in range(steps):
        Wg, Wu = (w.to(x.dtype) for w in master)
        z, kept = forward(x, Wg, Wu, Wd)
        diff = z - target
        losses.append(float(diff.square().mean()))
        for w, dw in zip(master, gradients((2.0 / diff.numel()) * diff, kept, Wg, Wu, Wd)):
            w -= rate * dw.float()
    return losses, [w.to(x.dtype) for w in master]


def serve(x, weights):
    """z of rows x on 4-bit weights, in x's type."""
    Wg, Wu, Wd = weights
    y, _, _ = api.exemplar_rmsnorm(x, eps=EPS)
    return x + api.exemplar_w4_product(api.exemplar_w4_glu(y, Wg, Wu), Wd)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--n", type=int, default=4096, help="rows")
    p.add_argument("--width", type=int, default=512)
    p.add_argument("--inner", type=int, default=1024, help="width inside the block")
    p.add_argument("--steps", type=int, default=8)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def block():
        return [(randn(a.inner, a.width) / a.width ** 0.5).bfloat16(), (randn(a.inner, a.width) / a.width ** 0.5).bfloat16(),
                (randn(a.width, a.inner) / a.inner ** 0.5).bfloat16()]

    x = randn(a.n, a.width).bfloat16()
    Wg, Wu, Wd = block()
    target, _ = forward(x, *(w + 0.3 * v for w, v in zip((Wg, Wu), block())), Wd)
    losses, (Wg, Wu) = train(x, target, Wg, Wu, Wd, a.steps, rate=0.25 * a.width)
    print("mean squared distance to the other block: " + " ".join("%.5f" % t for t in losses))

    weights = [api.exemplar_w4_quantize(w, 64) for w in (Wg, Wu, Wd)]
    bits = sum(8 * w.codes.numel() + 32 * w.words.numel() for w in weights) / (3 * a.width * a.inner)
    z, _ = forward(x, Wg, Wu, Wd)
    served = serve(x, weights)
    one = serve(x[:1], weights)
    off = float((served.float() - z).square().mean().sqrt() / z.square().mean().sqrt())
    print("served on weights of %.2f bits: off by %.3f of z; a single row by %.3f" % (
        bits, off, float((one.float() - z[:1]).square().mean().sqrt() / z[:1].square().mean().sqrt())))

    q, _, _ = api.exemplar_rmsnorm(served, eps=EPS, format=api.EXEMCL_MXFP4)
    sets = torch.randint(0, a.n, (64, 16), generator=g, device="cuda", dtype=torch.int32)
    f = api.exemplar_mx_eval(q, sets)
    print("best of 64 sets of exemplars: f %.4f, mean %.4f" % (float(f.max()), float(f.mean())))
    return losses, off, f


if __name__ == "__main__":
    main()
