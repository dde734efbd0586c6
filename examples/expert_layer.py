"""A layer of experts behind a cross-polytope hash: routed, trained in bf16, served from rotated 4-bit weights.

    python examples/expert_layer.py

Each vector goes to the expert that its bucket stands for (nearby vectors share buckets), vectors are sorted by expert, and each
expert multiplies its own rows.  Training takes both gradients of the grouped product; serving quantises the weights
once, after the rotation H D that spreads the inputs' few large coordinates, and the inputs on the way into each product.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1610_06209_amd import binding as sp  # noqa: E402


def route(x, signs, experts):
    """Order of the rows by expert, and where each expert's rows end."""
    bucket = sp.spinner_hash_signs(x, signs, 1)[:, 0].long() % experts
    order = torch.argsort(bucket, stable=True)
    return order, torch.cumsum(torch.bincount(bucket, minlength=experts), 0)


def main(rows=8192, n=2048, width=512, experts=16, steps=60, quiet=False):
    dev, gen = "cuda", torch.Generator(device="cuda")
    gen.manual_seed(1)
    # inputs with a few coordinates ten times as large as the others, in clusters; what is to be learned: a map of each expert's own
    centre = torch.randn((64, n), generator=gen, device=dev)
    x = centre[torch.randint(0, 64, (rows,), generator=gen, device=dev)] + 0.5 * torch.randn((rows, n), generator=gen, device=dev)
    x[:, torch.rand(n, generator=gen, device=dev) < 0.02] *= 10.0
    diag = (torch.randint(0, 2, (3, n), generator=gen, device=dev) * 2 - 1).float()
    order, ends = route(x, sp.spinner_pack_signs(diag[None]), experts)
    x = x[order].bfloat16()
    target = sp.spinner_grouped_matmul(x, (torch.randn((experts, width, n), generator=gen, device=dev) / math.sqrt(n)).bfloat16(), ends)

    # training: y = x w^T by expert, the gradient of its square error with respect to w in fp32
    w = torch.zeros((experts, width, n), device=dev)
    losses = []
    for _ in range(steps):
        w16 = w.bfloat16()
        error = sp.spinner_grouped_matmul(x, w16, ends) - target
        losses.append((error.float().square().mean() / target.float().square().mean()).item())
        dw = sp.spinner_grouped_matmul_dw(error, x, ends)
        # the step along dw that is best for each expert's square error: |dw|^2 over the square of what dw does to its rows
        line = sp.spinner_grouped_matmul(x, dw.bfloat16(), ends).double().square().sum(1)
        upto = torch.cat((line.new_zeros(1), line.cumsum(0)))
        curve = upto[ends] - upto[torch.cat((ends.new_zeros(1), ends[:-1]))]
        w -= (dw.flatten(1).double().square().sum(1) / curve.clamp_min(1e-30)).float()[:, None, None] * dw
    dx = sp.spinner_grouped_matmul_dx(error, w.bfloat16(), ends)                     # what the layer below would get

    def served(block):
        d = diag[0].contiguous() if block else None
        codes, scales = sp.spinner_mx_quantize(w.view(-1, n), d, block)
        y = sp.spinner_mx_linear(x, codes.view(experts, width, -1), scales.view(experts, width, -1), d, block, ends)
        return ((y - target).float().square().mean() / target.float().square().mean()).item()

    result = losses[0], losses[-1], served(n), served(0)
    one = sp.spinner_grouped_matmul(x[:1].contiguous(), w[:1].bfloat16())            # a single vector through one expert
    assert one.shape == (1, width) and dx.shape == x.shape
    if not quiet:
        print("relative square error: %.3f -> %.4f in bf16; 4 bits %.4f rotated, %.4f not rotated" % result)
    return result


if __name__ == "__main__":
    main()
