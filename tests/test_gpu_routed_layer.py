"""Router, order, ways there and back, products and 8-bit layers together, as a layer of experts uses them: values and gradients against a 64-bit model,
captured and replayed, on streams of their own, through the native part of the binding and without it."""
import os
import sys

import numpy as np
import pytest

from test_gpu_routing import gpu, numbers, say  # noqa: F401
from test_gpu_streams import check_call

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def inputs(g, rows, n, width, experts, seed=0):
    t = g.torch
    gen = t.Generator(device=g.dev)
    gen.manual_seed(seed)
    rand = lambda *s: t.randn(s, generator=gen, device=g.dev)      # noqa: E731
    return (rand(rows, n).bfloat16(), (rand(experts, n) * n ** -0.5).bfloat16(), (rand(experts, width, n) * n ** -0.5).bfloat16(),
            (rand(experts, n, width) * width ** -0.5).bfloat16(), 0.05 * rand(experts), rand(rows, n).bfloat16())


def model(t, x, router, up, down, chosen, scale):
    """The layer in 64 bits on the CPU for given choices, with torch's own gradients."""
    x, router, up, down = (a.double().cpu().requires_grad_() for a in (x, router, up, down))
    s = t.sigmoid(x @ router.T)
    out = t.zeros_like(x)
    picked = s.gather(1, chosen.clamp(min=0))
    w = t.where(chosen >= 0, picked, 0.0)
    w = scale * w / w.sum(1, keepdim=True).clamp_min(1e-300)
    for e in range(router.shape[0]):
        for j in range(chosen.shape[1]):
            at = (chosen[:, j] == e).nonzero()[:, 0]
            if len(at):
                out = out.index_add(0, at, w[at, j:j + 1] * ((x[at] @ up[e].T).relu() @ down[e].T))
    return out, (x, router, up, down)


@pytest.mark.parametrize("rows,n,width,experts,top", [(1, 64, 32, 8, 2), (37, 96, 40, 16, 4), (300, 128, 64, 12, 3), (1500, 64, 136, 64, 8)])
def test_a_layer_and_its_gradients(gpu, rows, n, width, experts, top):
    """Off by what bf16 takes from each of the six numbers that stand behind one another in a gradient: half a step of 2^-8 each at most, and less over a sum;
    3 % of the whole, in which a rectifier that switches at a rounding is small."""
    import routed_layer as layer

    say("routed layer", rows, n, width, experts, top)
    t = gpu.torch
    x, router, up, down, bias, dout = inputs(gpu, rows, n, width, experts)
    mask = t.arange(rows, device=gpu.dev) < max(1, rows - rows // 7)
    out, saved = layer.forward(x, router, up, down, bias, top, mask)
    grads = layer.backward(dout, x, router, up, down, saved)
    chosen = saved[2].long().cpu()
    assert (chosen[~mask.cpu()] == -1).all() and (chosen[mask.cpu()] >= 0).all()
    want, leaves = model(t, x, router, up, down, chosen, layer.ROUTER["scale"])
    want.backward(dout.double().cpu())
    for name, got, exact in zip(("out", "x", "router", "up", "down"), (out, *grads), (want, *(a.grad for a in leaves))):
        got, exact = got.double().cpu(), exact.detach()
        assert (got - exact).norm() <= 0.03 * exact.norm(), (name, float((got - exact).norm() / exact.norm()))
    assert (out[~mask] == 0).all() and (grads[0][~mask] == 0).all()


def test_gradient_of_the_weights_against_differences(gpu):
    """fp32 routers: the change of sum(dw . weights) over a small step of the logits, for choices that stay the same."""
    say("router differences")
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(3)
    x, d, step = (t.randn(s, generator=gen, device=gpu.dev, dtype=t.float64) for s in ((50, 40), (50, 6), (50, 40)))
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            weights, e = b.spinner_route(x.float(), 6, None, None, score, renormalise=renormalise)
            grad = b.spinner_route_grad(d.float(), x.float(), e, score, renormalise)
            h, total = 2.0 ** -7, []
            for sign in (1, -1):
                w, f = b.spinner_route((x + sign * h * step).float(), 6, None, None, score, renormalise=renormalise)
                # weights in the order of the first choices; rows that choose others are left out
                match = (e[:, :, None] == f[:, None, :])
                total.append((t.where(match, w.double()[:, None, :], 0.0).sum(2), match.any(2).all(1)))
            same = total[0][1] & total[1][1]
            got = ((total[0][0] - total[1][0]) * d).sum(1) / (2 * h)
            want = (grad.double() * step).sum(1)
            # h^2 / 6 of the third derivative, at most |d| |step|^3 sums of the scores, and fp32 weights over 2 h
            room = h * h * d.abs().sum(1) * step.abs().amax(1) ** 3 + d.abs().sum(1) * 2.0 ** -22 / h
            assert same.sum() > 20 and (((got - want).abs() <= room) | ~same).all()


def test_the_example_runs(gpu):
    import routed_layer as layer

    say("example")
    losses, off = layer.main(rows=512, n=512, width=256, experts=8, steps=3, quiet=True)
    assert len(losses) == 3 and np.isfinite(losses).all()
    # two layers of 8-bit inputs and weights: each off by about 1 / (127 sqrt(12)) of its row's largest number, four or five times the others'
    assert off < 0.05


def test_a_layer_captured_and_replayed(gpu):
    """A whole step, forward, back and served from 8 bits, in a graph: replays on new inputs in the same memory give the bits of the eager step."""
    import routed_layer as layer

    say("captured layer")
    t, b = gpu.torch, gpu.b
    rows, n, width, experts, top = 2100, 256, 128, 16, 4
    first = inputs(gpu, rows, n, width, experts)
    x, router, up, down, bias, dout = [a.clone() for a in first]
    d = [t.ones(n, device=gpu.dev), t.ones(width, device=gpu.dev)]
    packed = []
    for w in (up, down):
        c, s = b.spinner_int_quantize(w.view(-1, w.shape[2]), d[0] if w is up else d[1], 128)
        packed.append((c.view(experts, w.shape[1], -1), s.view(experts, -1)))

    def step():
        out, saved = layer.forward(x, router, up, down, bias, top)
        assert saved[2].numel() > 8192                                   # the order takes its two launches and a workspace
        return (out, *saved[:5], *layer.backward(dout, x, router, up, down, saved), layer.serve(x, router, *packed, bias, d, (128, 128), top))

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        step()
    t.cuda.current_stream().wait_stream(side)
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        held = step()
    for seed in range(4):
        for a, new in zip((x, router, up, down, bias, dout), inputs(gpu, rows, n, width, experts, seed)):
            a.copy_(new)
        for h in held:
            h.fill_(1)
        t.cuda.synchronize()
        want = step()
        graph.replay()
        t.cuda.synchronize()
        for h, e in zip(held, want):
            assert t.equal(h, e), seed


def calls(g):
    t, b = g.torch, g.b
    x, router, up, down, bias, dout = inputs(g, 2100, 256, 128, 16)
    logits = b.spinner_grouped_matmul(x, router)
    weights, chosen = b.spinner_route(logits, 4, bias)
    places, ends = b.spinner_route_order(chosen, 16)
    y = b.spinner_dispatch(x, places)
    d = t.ones(256, device=g.dev)
    codes, scales = b.spinner_int_quantize(x, d, 64)
    wc, ws = b.spinner_int_quantize(up.view(-1, 256), d, 64)
    wc, ws = wc.view(16, 128, -1), ws.view(16, 128)
    yc, ys = b.spinner_int_quantize(y, d, 64)
    t.cuda.synchronize()
    return {
        "route": lambda **k: b.spinner_route(logits, 4, bias, **k),
        "route_grad": lambda **k: b.spinner_route_grad(weights, logits, chosen, **k),
        "route_order": lambda **k: b.spinner_route_order(chosen, 16, **k),
        "dispatch": lambda **k: b.spinner_dispatch(x, places, **k),
        "combine": lambda **k: b.spinner_combine(y, places, weights, **k),
        "combine_grad": lambda **k: b.spinner_combine_grad(dout, y, places, weights, **k),
        "int_quantize": lambda **k: b.spinner_int_quantize(x, d, 64, places, **k),
        "int_dequantize": lambda **k: b.spinner_int_dequantize(codes, scales, t.bfloat16, **k),
        "int_matmul": lambda **k: b.spinner_int_matmul(yc, ys, wc, ws, ends, **k),
        "int_linear": lambda **k: b.spinner_int_linear(x, wc, ws, d, 64, ends, places, **k),
    }


CALLS = ["route", "route_grad", "route_order", "dispatch", "combine", "combine_grad", "int_quantize", "int_dequantize", "int_matmul", "int_linear"]


@pytest.mark.parametrize("name", CALLS)
def test_calls_on_a_stream_of_their_own(gpu, name, monkeypatch):
    say("stream of its own", name)
    check_call(gpu, calls(gpu)[name], monkeypatch)


@pytest.mark.parametrize("name", CALLS)
def test_native_calls_give_the_bits_of_the_long_way(gpu, name, monkeypatch):
    """The native part answers the usual call itself; without it the binding gives the same bits."""
    say("native", name)
    t, b = gpu.torch, gpu.b
    call, asked = calls(gpu)[name], []

    class Native:
        def __init__(self, served):
            self.served = served

        def __getattr__(self, which):
            def f(*a):
                r = getattr(real, which)(*a) if self.served else None
                asked.append((which, r is not None))
                return r
            return f

    real = b._native_experts
    monkeypatch.setattr(b, "_native_experts", Native(True))
    one = call()
    monkeypatch.setattr(b, "_native_experts", Native(False))
    two = call()
    assert asked == [(name, True), (name, False)]
    pairs = list(zip(one, two)) if isinstance(one, tuple) else [(one, two)]
    assert all(p.dtype == q.dtype and t.equal(p, q) for p, q in pairs)
    # what is out of the ordinary is left to the long way: streams, tensors of the host
    monkeypatch.setattr(b, "_native_experts", Native(True))
    asked.clear()
    call(stream=t.cuda.current_stream())
    assert asked == [(name, False)]


def test_calls_side_by_side(gpu):
    """Two orders and two layers at once on streams of their own, each with memory of its own."""
    say("side by side")
    t, b = gpu.torch, gpu.b
    made = calls(gpu)
    want = {k: made[k]() for k in ("route_order", "int_linear", "route")}
    t.cuda.synchronize()
    streams = [t.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(5):
        for s in streams:
            with t.cuda.stream(s):
                got.append({k: made[k]() for k in want})
    t.cuda.synchronize()
    for g in got:
        for k, w in want.items():
            for p, q in zip(g[k] if isinstance(w, tuple) else (g[k],), w if isinstance(w, tuple) else (w,)):
                assert t.equal(p, q)


def test_a_workspace_of_the_callers(gpu):
    say("workspaces")
    t, b = gpu.torch, gpu.b
    e = t.randint(0, 40, (20000, 3), dtype=t.int32, device=gpu.dev)
    need = b.spinner_route_order_workspace_bytes(e.numel(), 40)
    scratch = t.full((need,), 255, dtype=t.uint8, device=gpu.dev)
    for p, q in zip(b.spinner_route_order(e, 40, workspace=scratch), b.spinner_route_order(e, 40)):
        assert t.equal(p, q)
    x, w = t.randn((70, 300), device=gpu.dev).bfloat16(), t.randn((33, 300), device=gpu.dev)
    wc, ws = b.spinner_int_quantize(w)
    need = b.spinner_int_linear_workspace_bytes(70, 300)
    scratch = t.full((need,), 255, dtype=t.uint8, device=gpu.dev)
    assert t.equal(b.spinner_int_linear(x, wc, ws, workspace=scratch), b.spinner_int_linear(x, wc, ws))
    with pytest.raises(ValueError):
        b.spinner_int_linear(x, wc, ws, workspace=scratch[:-1])
    # a few rows need none
    for rows, status in ((4, b.SPINNER_OK), (5, b.SPINNER_ERR_WORKSPACE)):
        x, wc, ws = t.randn((rows, 1024), device=gpu.dev).bfloat16(), *b.spinner_int_quantize(t.randn((48, 1024), device=gpu.dev))
        out = t.full((rows, 48), 5.0, device=gpu.dev).bfloat16()
        rc = b.lib.spinner_int_linear(x.data_ptr(), 1, rows, 1024, 1024, None, 0, None, 1, wc.data_ptr(), ws.data_ptr(), 48, 1, None, out.data_ptr(), 48, None,
                                      b._stream_handle(None))
        assert rc == status and (t.equal(out, b.spinner_int_linear(x, wc, ws)) if rc == b.SPINNER_OK else bool((out == 5).all()))
