"""A feed-forward block that trains with microscaled 4-bit operands: norm with the residual's addition, two linear layers, and back.

    python examples/train_block.py [--tokens 512] [--steps 20]

Every matrix is quantised where a product needs it: along its rows for the product itself, down its columns for the product of a gradient, both
from one read.  Gradients are rounded stochastically, each step by another seed.  Weights stay in FP32 and take plain gradient steps.  The last
line compares the first step's gradients with those of the same block in FP32.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1804_01526_amd import hbfp  # noqa: E402

EPS = 1e-5


class Block:
    """y = silu(norm(x + residual) w1^T) w2^T, added to the residual stream."""

    def __init__(self, features, hidden, gen):
        def randn(*shape):
            return torch.randn(shape, generator=gen, device="cuda")
        self.weight = torch.ones(features, device="cuda")
        self.w1, self.w2 = randn(hidden, features) / math.sqrt(features), randn(features, hidden) / math.sqrt(hidden)

    def forward(self, x, residual):
        normed, total, rstd, values = hbfp.norm_mx4(x, self.weight, EPS, residual=residual, values=True)
        (w1, w1_down), (w2, w2_down) = hbfp.quant_mx4_both(self.w1), hbfp.quant_mx4_both(self.w2)
        h = hbfp.gemm_mx4(normed, w1)
        gate = torch.sigmoid(h)
        h_along, h_down = hbfp.quant_mx4_both(h * gate)
        y = hbfp.gemm_mx4(h_along, w2, dtype=x.dtype)
        # kept for the way back: 4.25 bits a value where that is enough
        self.kept = total, rstd, hbfp.quant_mx4(values, axis=0), gate * (1 + h * (1 - gate)), h_down, w1_down, w2_down
        return total + y

    def backward(self, g, seed):
        """g: the gradient of what forward returned.  Returns that of x (and of the residual) and of the three parameters."""
        total, rstd, values_down, slope, h_down, w1_down, w2_down = self.kept
        g_along, g_down = hbfp.quant_mx4_both(g, hbfp.STOCHASTIC, 2 * seed)
        dw2 = hbfp.gemm_mx4(g_down, h_down)
        dh = hbfp.gemm_mx4(g_along, w2_down) * slope
        dh_along, dh_down = hbfp.quant_mx4_both(dh, hbfp.STOCHASTIC, 2 * seed + 1)
        dw1 = hbfp.gemm_mx4(dh_down, values_down)
        dn = hbfp.gemm_mx4(dh_along, w1_down, dtype=g.dtype)
        dx, dweight = hbfp.norm_grad(dn, total, rstd, self.weight, g_sum=g)
        return dx, dweight, dw1, dw2


def plain(block, x, residual, g):
    """The same in FP32, by autograd."""
    leaves = [t.detach().float().requires_grad_() for t in (x, block.weight, block.w1, block.w2)]
    total = leaves[0] + residual.float()
    n = total * torch.rsqrt((total * total).mean(dim=1, keepdim=True) + EPS) * leaves[1]
    y = total + torch.nn.functional.silu(n @ leaves[2].t()) @ leaves[3].t()
    y.backward(g.float())
    return y.detach(), [t.grad for t in leaves]


def inputs(tokens, features, dtype, gen):
    return [torch.randn((tokens, features), generator=gen, device="cuda").to(dtype) for _ in range(3)]


def compare(tokens=512, features=512, hidden=1024, dtype=torch.bfloat16, seed=0):
    """Relative errors of the output and of the gradients of x, norm weight, w1 and w2 against FP32."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    block = Block(features, hidden, gen)
    x, residual, g = inputs(tokens, features, dtype, gen)
    got = [block.forward(x, residual), *block.backward(g, seed + 1)]
    y, grads = plain(block, x, residual, g)
    return [float((a.float() - b).norm() / b.norm()) for a, b in zip(got, [y, *grads])]


def run(tokens=512, steps=20, features=512, hidden=1024, rate=0.5, seed=0):
    """A few steps towards a fixed output; the mean square distance before each."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    block = Block(features, hidden, gen)
    x, residual, target = inputs(tokens, features, torch.bfloat16, gen)
    losses = []
    for step in range(steps):
        y = block.forward(x, residual)
        off = y.float() - target.float()
        losses.append(float(off.square().mean()))
        _, dweight, dw1, dw2 = block.backward((off * (2.0 / off.numel())).bfloat16(), step)
        for parameter, gradient in ((block.weight, dweight), (block.w1, dw1), (block.w2, dw2)):
            parameter -= rate * gradient
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--tokens", type=int, default=512)
    parser.add_argument("--steps", type=int, default=20)
    args = parser.parse_args()
    losses = run(args.tokens, args.steps)
    print(f"{args.steps} steps on {args.tokens} tokens: mean square distance {losses[0]:.3f} -> {losses[-1]:.3f}")
    names = ("output", "x", "norm weight", "w1", "w2")
    print("relative error against FP32: " + ", ".join(f"{n} {e:.3f}" for n, e in zip(names, compare(args.tokens))))
