"""Products of rows grouped by expert in 16 bits, and their gradients, against 64-bit products (oracle/mx4_oracle.py).

Tolerances: products of 16-bit numbers are exact in fp32 (bf16; fp16 in fp32's range), a sum passes through at most
depth / 16 + 16 additions of the matrix pipe, each off by at most 2^-23 of the sum of magnitudes, and is rounded once."""
import sys

import numpy as np
import pytest

from oracle import mx4_oracle as mx

pytestmark = pytest.mark.gpu
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -140, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1610_06209_amd import binding

    class G:
        pass

    g = G()
    g.torch, g.b, g.dev = torch, binding, torch.device("cuda:0")
    g.types = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    return g


def say(*a):
    print("\n[gpu-case]", *a, file=sys.stderr, flush=True)


def held(g, x, name):
    t = g.torch.from_numpy(np.ascontiguousarray(x)).to(g.types[name]).to(g.dev)
    return t, t.double().cpu().numpy()


def numbers(t):
    return t.double().cpu().numpy()


def check(got, want, size, depth, out):
    bound = np.abs(want) * 1.01 * HALF_STEP[out] + size * (depth / 16 + 16) * 2.0 ** -23 + TINY[out]
    off = np.abs(got - want)
    assert np.all(off <= bound), float((off / bound).max())


def ragged(rng, rows, experts, spare=0):
    ends = np.concatenate((np.sort(rng.integers(0, rows - spare + 1, experts - 1)), [rows - spare]))
    if experts > 3:
        ends[1] = ends[0]
    return np.maximum.accumulate(ends).astype(np.int64)


SIZES = [(1, 8, 8, 1), (1, 2048, 100, 2), (5, 1, 1, 2), (24, 256, 129, 8), (40, 72, 64, 3), (64, 136, 200, 1), (100, 33, 7, 5), (130, 64, 128, 2),
         (200, 1000, 130, 64), (257, 256, 256, 1), (500, 100, 60, 65), (700, 129, 257, 4), (900, 520, 264, 3), (1500, 128, 384, 200)]


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n,experts", SIZES)
def test_products_and_gradients(gpu, name, rows, k, n, experts):
    say("grouped", name, rows, k, n, experts)
    rng = np.random.default_rng(rows + k + n + experts)
    x, xe = held(gpu, rng.standard_normal((rows, k)), name)
    dy, dye = held(gpu, rng.standard_normal((rows, n)), name)
    w, we = held(gpu, rng.standard_normal((experts, n, k)), name)
    every = [ragged(rng, rows, experts), ragged(rng, rows, experts, rows // 4), rng.integers(-5, rows + 5, experts)]
    for ends in every + ([None] if experts == 1 else []):
        e = None if ends is None else gpu.torch.from_numpy(ends).to(gpu.dev)
        y = numbers(gpu.b.spinner_grouped_matmul(x, w, e))
        check(y, mx.products(xe, we, ends), mx.products(np.abs(xe), np.abs(we), ends), k, name)
        dx = numbers(gpu.b.spinner_grouped_matmul_dx(dy, w, e))
        check(dx, mx.products_dx(dye, we, ends), mx.products_dx(np.abs(dye), np.abs(we), ends), n, name)
        last = 0 if ends is None else mx.bounds(ends, experts, rows)[-1][1]
        if ends is not None:
            assert not y[last:].any() and not dx[last:].any()
        want, size = mx.products_dw(dye, xe, experts, ends), mx.products_dw(np.abs(dye), np.abs(xe), experts, ends)
        for out in ("f32", name):
            dw = numbers(gpu.b.spinner_grouped_matmul_dw(dy, x, e, gpu.types[out]))
            check(dw.reshape(want.shape), want, size, rows, out)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n,experts", [(30, 40, 24, 4), (600, 200, 136, 3), (200, 35, 51, 6)])
def test_gradients_are_those_of_differences(gpu, name, rows, k, n, experts):
    """Small whole numbers and steps of 1: every sum is exact in the type of the results, so the differences are too."""
    say("gradients by differences", name, rows, k, n, experts)
    t, rng = gpu.torch, np.random.default_rng(k)
    few = lambda *s: np.where(rng.random(s) < 24.0 / max(s[-1], 24), rng.integers(-1, 2, s), 0).astype(float)     # noqa: E731
    x, xe = held(gpu, few(rows, k), name)
    w, we = held(gpu, few(experts, n, k), name)
    dy, dye = held(gpu, few(rows, n), name)
    ends = t.from_numpy(ragged(rng, rows, experts, 2)).to(gpu.dev)
    u, v = few(rows, k), few(experts, n, k)
    loss = lambda a, b: float((dye * numbers(gpu.b.spinner_grouped_matmul(held(gpu, a, name)[0], held(gpu, b, name)[0], ends))).sum())  # noqa: E731
    dx, dw = gpu.b.spinner_grouped_matmul_dx(dy, w, ends), gpu.b.spinner_grouped_matmul_dw(dy, x, ends)
    assert (loss(xe + u, we) - loss(xe - u, we)) / 2 == float((numbers(dx) * u).sum())
    assert (loss(xe, we + v) - loss(xe, we - v)) / 2 == float((numbers(dw) * v).sum())


@pytest.mark.parametrize("k,n", [(64, 40), (61, 43)])
def test_strides_and_results_in_wider_rows(gpu, k, n):
    say("grouped: strides", k, n)
    t, rng = gpu.torch, np.random.default_rng(3)
    rows, experts = 150, 3
    xb, _ = held(gpu, rng.standard_normal((rows, k + 3)), "bf16")
    dyb, _ = held(gpu, rng.standard_normal((rows, n + 8)), "bf16")
    w, _ = held(gpu, rng.standard_normal((experts, n, k)), "bf16")
    ends = t.tensor([100, 100, 147], device=gpu.dev)
    for x, dy in ((xb[:, :k], dyb[:, :n]), (xb[:1, :k].expand(rows, k), dyb[:1, :n].expand(rows, n))):
        xc, dyc = x.contiguous(), dy.contiguous()
        assert t.equal(gpu.b.spinner_grouped_matmul(x, w, ends), gpu.b.spinner_grouped_matmul(xc, w, ends))
        assert t.equal(gpu.b.spinner_grouped_matmul_dx(dy, w, ends), gpu.b.spinner_grouped_matmul_dx(dyc, w, ends))
        assert t.equal(gpu.b.spinner_grouped_matmul_dw(dy, x, ends), gpu.b.spinner_grouped_matmul_dw(dyc, xc, ends))
        out = t.full((rows, n + 5), 3.0, dtype=t.bfloat16, device=gpu.dev)
        gpu.b.spinner_grouped_matmul(x, w, ends, out[:, :n])
        assert t.equal(out[:, :n], gpu.b.spinner_grouped_matmul(xc, w, ends)) and bool((out[:, n:] == 3).all())
        dx = t.full((rows, k + 1), 3.0, dtype=t.bfloat16, device=gpu.dev)
        gpu.b.spinner_grouped_matmul_dx(dy, w, ends, dx[:, :k])
        assert t.equal(dx[:, :k], gpu.b.spinner_grouped_matmul_dx(dyc, w, ends)) and bool((dx[:, k:] == 3).all())


@pytest.mark.parametrize("rows", [9, 100, 600])
@pytest.mark.parametrize("k,n", [(64, 72), (63, 70)])
def test_no_number_stays_with_its_expert(gpu, rows, k, n):
    """NaN and infinities in another expert's rows, in rows of none, in another expert's weights: results as without them."""
    say("grouped: NaN", rows, k, n)
    t, rng = gpu.torch, np.random.default_rng(3)
    x, _ = held(gpu, rng.standard_normal((rows, k)), "bf16")
    dy, _ = held(gpu, rng.standard_normal((rows, n)), "bf16")
    w, _ = held(gpu, rng.standard_normal((3, n, k)), "bf16")
    mid, last = rows // 2, rows - 3
    ends = t.tensor([mid, last, last], device=gpu.dev)
    calls = [lambda x, dy, w: gpu.b.spinner_grouped_matmul(x, w, ends), lambda x, dy, w: gpu.b.spinner_grouped_matmul_dx(dy, w, ends),
             lambda x, dy, w: gpu.b.spinner_grouped_matmul_dw(dy, x, ends)]
    clean = [c(x, dy, w) for c in calls]
    x2, dy2, w2 = x.clone(), dy.clone(), w.clone()
    x2[mid:] = float("nan")
    dy2[mid:] = float("inf")
    w2[1:] = float("nan")
    bad = [c(x2, dy2, w2) for c in calls]
    for a, b in zip(clean[:2], bad[:2]):
        assert t.equal(a[:mid], b[:mid]) and not bool(b[last:].any()) and not bool(b[mid:last].isfinite().any())
    assert t.equal(clean[2][0], bad[2][0]) and not bool(bad[2][2].any()) and bool(bad[2][1].isnan().all())


def test_empty_and_refused(gpu):
    say("grouped: empty, refusals")
    t, b = gpu.torch, gpu.b
    x, dy, w = (t.zeros(s, dtype=t.bfloat16, device=gpu.dev) for s in ((6, 16), (6, 8), (2, 8, 16)))
    ends = t.tensor([2, 6], device=gpu.dev)
    assert b.spinner_grouped_matmul(x[:0], w, ends).shape == (0, 8) and b.spinner_grouped_matmul_dx(dy[:0], w, ends).shape == (0, 16)
    dw = t.full((2, 8, 16), 4.0, device=gpu.dev)
    b.spinner_grouped_matmul_dw(dy[:0], x[:0], ends, t.float32, dw)
    assert not bool(dw.any())
    for call in (lambda: b.spinner_grouped_matmul(x.float(), w.float(), ends), lambda: b.spinner_grouped_matmul_dx(dy.float(), w.float(), ends),
                 lambda: b.spinner_grouped_matmul_dw(dy.float(), x.float(), ends), lambda: b.spinner_grouped_matmul_dw(dy, x, ends, t.float16)):
        with pytest.raises(b.SpinnerError) as e:
            call()
        assert e.value.status == b.SPINNER_ERR_BAD_TYPE
    for bad in (lambda: b.spinner_grouped_matmul(x, w.half(), ends), lambda: b.spinner_grouped_matmul(x, w), lambda: b.spinner_grouped_matmul(dy, w, ends),
                lambda: b.spinner_grouped_matmul(x, w.transpose(1, 2), ends), lambda: b.spinner_grouped_matmul(x, w, ends.float()),
                lambda: b.spinner_grouped_matmul(x, w, ends, x), lambda: b.spinner_grouped_matmul_dw(dy, x[:3], ends),
                lambda: b.spinner_grouped_matmul_dw(dy, x, ends, t.float32, w), lambda: b.spinner_grouped_matmul(x.cpu(), w, ends)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(b.SpinnerError) as e:
        b.spinner_grouped_matmul(x.reshape(-1)[1:81].view(5, 16), w, ends)
    assert e.value.status == b.SPINNER_ERR_ALIGNMENT
    many = t.zeros((1025, 1, 8), dtype=t.bfloat16, device=gpu.dev)
    with pytest.raises(b.SpinnerError) as e:
        b.spinner_grouped_matmul(x[:, :8].contiguous(), many, t.zeros(1025, dtype=t.int64, device=gpu.dev))
    assert e.value.status == b.SPINNER_ERR_BAD_SHAPE


def test_both_ways_of_a_call_streams_and_graph(gpu):
    say("grouped: native and long way, streams, graph")
    t, b, rng = gpu.torch, gpu.b, np.random.default_rng(1)
    x, _ = held(gpu, rng.standard_normal((200, 96)), "f16")
    dy, _ = held(gpu, rng.standard_normal((200, 80)), "f16")
    w, _ = held(gpu, rng.standard_normal((3, 80, 96)), "f16")
    ends = t.tensor([60, 60, 190], device=gpu.dev)
    calls = [lambda o=None, **k: b.spinner_grouped_matmul(x, w, ends, o, **k), lambda o=None, **k: b.spinner_grouped_matmul_dx(dy, w, ends, o, **k),
             lambda o=None, **k: b.spinner_grouped_matmul_dw(dy, x, ends, t.float16, o, **k)]
    side = t.cuda.Stream()
    first = [c() for c in calls]
    side.wait_stream(t.cuda.current_stream())
    other = [c(stream=side) for c in calls]
    side.synchronize()
    assert all(t.equal(p, q) for p, q in zip(first, other))
    outs = [t.zeros_like(f) for f in first]
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        for c, o in zip(calls, outs):
            c(o)
    for k in range(4):
        x.copy_(t.from_numpy(rng.standard_normal((200, 96))).to(x.dtype))
        ends.copy_(t.tensor([50 + 9 * k, 120, 200 - k]))
        for o in outs:
            o.zero_()
        graph.replay()
        t.cuda.synchronize()
        assert all(t.equal(o, c()) for c, o in zip(calls, outs))


def test_places_beyond_32_bits(gpu):
    say("grouped: offsets beyond 32 bits")
    t, b = gpu.torch, gpu.b
    rows, k, n = (1 << 21) + 200, 1032, 1040               # 2.2e9 numbers in and out
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(1)
    part = t.randn((1 << 14, k), generator=gen, device=gpu.dev).to(t.bfloat16)
    x = part.repeat((rows >> 14) + 1, 1)[:rows]
    w = t.randn((2, n, k), generator=gen, device=gpu.dev).to(t.bfloat16)
    at = (rows >> 14) << 14
    ends = t.tensor([at - (1 << 14), rows], device=gpu.dev)
    y = b.spinner_grouped_matmul(x, w, ends)
    want = b.spinner_grouped_matmul(part[: rows - at].clone(), w[1].contiguous())
    assert t.allclose(y[at:].float(), want.float(), rtol=2.0 ** -7, atol=1e-2)
    dx = b.spinner_grouped_matmul_dx(y, w, ends)
    want = b.spinner_grouped_matmul_dx(y[at:].clone(), w[1].contiguous())
    assert t.allclose(dx[at:].float(), want.float(), rtol=2.0 ** -7, atol=1.0)
    dw = b.spinner_grouped_matmul_dw(y, x, ends)
    want = b.spinner_grouped_matmul_dw(y[at - (1 << 14):].clone(), x[at - (1 << 14):].clone())
    assert t.allclose(dw[1], want, rtol=1e-3, atol=1e-3 * float(want.abs().max()))
