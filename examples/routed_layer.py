"""A layer of experts behind a learned router: routed by score, trained in bf16 with every gradient, served from rotated 8-bit weights.

    python examples/routed_layer.py

Each vector goes to the few experts that its router scores highest (sigmoid scores, a bias that keeps the load even, groups of
experts of which some stay), through two products with a rectifier between them, and back as a weighted sum.  The step back takes the
same way: through the sum to the experts and the weights, through the products, and through the router to its own weights.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1610_06209_amd import binding as sp  # noqa: E402

ROUTER = dict(score="sigmoid", groups=4, top_groups=2, group_top=2, renormalise=True, scale=1.5)


def forward(x, router, up, down, bias, top=4, mask=None):
    """The layer's output, and what the way back needs."""
    logits = sp.spinner_grouped_matmul(x, router)
    weights, chosen = sp.spinner_route(logits, top, bias, mask, **ROUTER)
    places, ends = sp.spinner_route_order(chosen, router.shape[0])
    xs = sp.spinner_dispatch(x, places)
    h = sp.spinner_grouped_matmul(xs, up, ends)
    a = h.relu()
    y = sp.spinner_grouped_matmul(a, down, ends)
    return sp.spinner_combine(y, places, weights), (logits, weights, chosen, places, ends, xs, h, a, y)


def backward(dout, x, router, up, down, saved):
    """Gradients with respect to x (of its type) and to the router's and experts' weights (fp32)."""
    logits, weights, chosen, places, ends, xs, h, a, y = saved
    dy, dweights = sp.spinner_combine_grad(dout, y, places, weights)
    ddown = sp.spinner_grouped_matmul_dw(dy, a, ends)
    dh = sp.spinner_grouped_matmul_dx(dy, down, ends) * (h > 0)
    dup = sp.spinner_grouped_matmul_dw(dh, xs, ends)
    dx = sp.spinner_combine(sp.spinner_grouped_matmul_dx(dh, up, ends), places)
    dlogits = sp.spinner_route_grad(dweights, logits, chosen, ROUTER["score"], ROUTER["renormalise"], ROUTER["scale"])
    dx = dx + sp.spinner_grouped_matmul_dx(dlogits, router)
    return dx, sp.spinner_grouped_matmul_dw(dlogits, x), dup, ddown


def rebalance(bias, ends, rate=0.02):
    """Experts with more rows than the mean become harder to choose, those with fewer easier."""
    load = torch.diff(ends, prepend=ends.new_zeros(1)).float()
    return bias - rate * torch.sign(load - load.mean())


def serve(x, router, up8, down8, bias, diag, block, top=4):
    """The layer from 8-bit experts: each row is rotated and rounded once on its way to its experts."""
    weights, chosen = sp.spinner_route(sp.spinner_grouped_matmul(x, router), top, bias, **ROUTER)
    places, ends = sp.spinner_route_order(chosen, router.shape[0])
    h = sp.spinner_int_linear(x, *up8, diag[0], block[0], ends, places)
    y = sp.spinner_int_linear(h.relu_(), *down8, diag[1], block[1], ends)
    return sp.spinner_combine(y, places, weights)


def main(rows=4096, n=1024, width=512, experts=16, steps=40, quiet=False):
    dev, gen = "cuda", torch.Generator(device="cuda")
    gen.manual_seed(1)
    rand = lambda *shape, scale=1.0: scale * torch.randn(shape, generator=gen, device=dev)      # noqa: E731
    x = (rand(64, n)[torch.randint(0, 64, (rows,), generator=gen, device=dev)] + 0.3 * rand(rows, n)).bfloat16()
    teacher = [rand(experts, n, scale=n ** -0.5), rand(experts, width, n, scale=n ** -0.5), rand(experts, n, width, scale=width ** -0.5)]
    bias = torch.zeros(experts, device=dev)
    target = forward(x, *[w.bfloat16() for w in teacher], bias)[0].float()
    w = [t + rand(*t.shape, scale=0.3 / math.sqrt(t.shape[-1])) for t in teacher]
    losses = []
    for _ in range(steps):
        w16 = [t.bfloat16() for t in w]
        out, saved = forward(x, *w16, bias)
        error = out.float() - target
        losses.append((error.square().mean() / target.square().mean()).item())
        grads = backward(error.bfloat16(), x, *w16, saved)[1:]
        for t, g, rate in zip(w, grads, (0.02, 0.3, 0.3)):
            t -= rate * g / g.square().mean().sqrt().clamp_min(1e-30) * t.square().mean().sqrt() * 0.05
        bias = rebalance(bias, saved[4], 1e-3)
    w16 = [t.bfloat16() for t in w]
    direct = forward(x, *w16, bias)[0]
    # served: both matrices of each expert rotated along their inputs and rounded to 8 bits once
    diag = [(torch.randint(0, 2, (k,), generator=gen, device=dev) * 2 - 1).float() for k in (n, width)]
    block = [512, width]
    packed = []
    for t, d, b in zip(w16[1:], diag, block):
        codes, scales = sp.spinner_int_quantize(t.view(-1, t.shape[2]), d, b)
        packed.append((codes.view(experts, t.shape[1], -1), scales.view(experts, -1)))
    served = serve(x, w16[0], *packed, bias, diag, block)
    off = ((served - direct).float().square().mean() / direct.float().square().mean()).sqrt().item()
    one = serve(x[:1].contiguous(), w16[0], *packed, bias, diag, block)                          # a single vector
    assert one.shape == (1, n)
    if not quiet:
        print("relative square error: %.4f -> %.4f; 8-bit weights differ from bf16 by %.4f" % (losses[0], losses[-1], off))
    return losses, off


if __name__ == "__main__":
    main()
