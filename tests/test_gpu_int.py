"""Layers of 8-bit whole numbers against the 64-bit definitions (oracle/experts_oracle.py).

Tolerances.  Without a rotation scales and codes are the definition's, exactly.  Rotated numbers pass through log2(block) butterflies and the diagonal's
factor in fp32, each off by at most 2^-24 of what may be as large as the run's norm; a code then is off by half a step, that, and the 2e-5 of a step
that the product with the rounded 1 / scale may take.  Products: whole sums are exact, then a rounding to fp32, two factors and a rounding to the type."""
import sys

import numpy as np
import pytest

from oracle import experts_oracle as ex
from oracle import mx4_oracle as mx
from test_gpu_routing import HALF_STEP, TINY, gpu, held, numbers  # noqa: F401

pytestmark = pytest.mark.gpu


def say(*a):
    print("\n[gpu-case]", *a, file=sys.stderr, flush=True)


def width(k):
    return -(-k // 16) * 16


def whole(codes, k):
    """Codes as the definition has them; the padding is zeros."""
    c = codes.cpu().numpy().astype(np.int64)
    assert c.shape[-1] == width(k) and not c[..., k:].any()
    return c[..., :k]


WIDTHS = [1, 7, 8, 15, 16, 17, 100, 511, 512, 513, 1000, 2047, 2048, 2056, 4095, 4097, 8192, 10007, 16384, 16400, 40001, 131056]


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", WIDTHS)
def test_rounding_without_a_rotation(gpu, name, k):
    say("int quantise", name, k)
    rng = np.random.default_rng(k)
    rows = 37 if k < 5000 else 5
    x = rng.standard_normal((rows, k)) * np.exp(3 * rng.standard_normal((rows, 1)))
    x[1] = 0
    x[2, rng.integers(0, k)] = 300.0                       # an outlier, or all there is
    x[3] = np.rint(x[3] * 4) / 2
    x[3, 0] = 127 / 2                                      # scale 1 / 2: many ties
    xt, xe = held(gpu, x, name)
    codes, scales = gpu.b.spinner_int_quantize(xt)
    want, want_s = ex.int_quantize(xe)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(whole(codes, k), want)
    for out in ("f32", "bf16", "f16"):
        got, exact = numbers(gpu.b.spinner_int_dequantize(codes, scales, gpu.types[out], k)), want * want_s.astype(np.float64)[:, None]
        assert np.all(np.abs(got - exact) <= np.abs(exact) * 1.01 * (HALF_STEP[out] + 2.0 ** -24) + TINY[out])


def test_values_that_are_no_ordinary_numbers(gpu):
    """NaN and infinities, the smallest and the largest numbers, and what they do to products."""
    say("int values")
    t = gpu.torch
    x = np.zeros((9, 40), dtype=np.float32)
    x[0, 3], x[1, 4], x[2, 5] = np.nan, np.inf, -np.inf
    x[3] = 2.0 ** -149
    x[4, ::2] = 2.0 ** -126 * 3
    x[5] = np.finfo(np.float32).max
    x[6, 1] = -1e-38
    x[7, :5] = [np.float32(127 * 2.0 ** -126), 2.0 ** -126, 2.0 ** -127, 3 * 2.0 ** -127, -5 * 2.0 ** -127]
    x[8] = -0.0
    xt, xe = held(gpu, x)
    codes, scales = gpu.b.spinner_int_quantize(xt)
    want, want_s = ex.int_quantize(xe)
    assert np.array_equal(scales.cpu().numpy(), want_s, equal_nan=True) and np.array_equal(whole(codes, 40), want)
    w, ws = gpu.b.spinner_int_quantize(t.randn((50, 40), device=gpu.dev))
    # NaN for the rows that are not finite; the row of the largest number leaves fp32's range with some weights
    exact = ex.int_products(want, want_s, whole(w, 40)[None], ws.cpu().numpy()[None])
    beyond = np.abs(exact) > np.finfo(np.float32).max

    def fits(y, r):
        return t.isnan(y).all() if r < 3 else np.array_equal(t.isinf(y).cpu().numpy(), beyond[r]) and not t.isnan(y).any()

    for rows in (9, 40):                                   # the form for few rows, and tiles
        c, s = codes.repeat(5, 1)[:rows].contiguous(), scales.repeat(5)[:rows].contiguous()
        y = gpu.b.spinner_int_matmul(c, s, w, ws, dtype=t.float32)
        for r in range(rows):
            assert fits(y[r], r % 9)
    y = gpu.b.spinner_int_linear(xt, w, ws)
    assert all(fits(y[r], r) for r in range(9))


ROTATED = [(32, 32), (96, 32), (512, 64), (640, 128), (768, 256), (1024, 512), (2048, 1024), (1536, 512), (4096, 2048), (6144, 2048), (4096, 4096), (8192, 4096), (20480, 4096), (36864, 1024), (24576, 4096)]


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k,block", ROTATED)
def test_rounding_after_a_rotation(gpu, name, k, block):
    say("int rotate", name, k, block)
    rng = np.random.default_rng(k + block)
    rows = 6
    x, xe = held(gpu, rng.standard_normal((rows, k)) * np.where(rng.random(k) < 0.02, 20.0, 1.0), name)
    d, de = held(gpu, rng.standard_normal(k))
    for diag, dx in ((d, de), (None, None)):
        v = mx.rotate(xe, dx, block)
        codes, scales = gpu.b.spinner_int_quantize(x, diag, block)
        s = scales.double().cpu().numpy()[:, None]
        runs = (xe * (1 if dx is None else dx)).reshape(rows, -1, block)
        norm = np.repeat(np.linalg.norm(runs, axis=-1), block, -1).reshape(rows, k)
        off = (np.log2(block) + 3) * 2.0 ** -24 * norm
        assert np.all(np.abs(s[:, 0] - np.abs(v).max(1) / 127) <= off.max(1) / 127 + np.abs(v).max(1) / 127 * 2.0 ** -23)
        assert np.all(np.abs(whole(codes, k) * s - v) <= s * (0.5 + 3e-5) + off)
        assert np.abs(whole(codes, k)).max() == 127


MANY = [(5000, 0), (4112, 0), (7680, 32), (8192, 64), (4608, 128), (4352, 256), (5120, 512), (6144, 1024), (8192, 2048), (8192, 4096), (1536, 512), (400, 0), (18432, 1024)]


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k,block", MANY)
def test_many_rows_have_the_bits_of_few(gpu, name, k, block):
    """Rows a workgroup takes in turn, and the forms that only many rows take: codes and scales as of a few rows at a time."""
    say("int many rows", name, k, block)
    t = gpu.torch
    rows = 9001
    g = t.Generator(device=gpu.dev).manual_seed(k)
    x = (t.randn((rows, k), device=gpu.dev, generator=g) * t.exp(t.randn((rows, 1), device=gpu.dev, generator=g))).to(gpu.types[name])
    d = t.sign(t.randn(k, device=gpu.dev, generator=g)) if block else None
    codes, scales = gpu.b.spinner_int_quantize(x, d, block)
    for r0 in (0, 500, 1020, 2000, 4093, 8190, rows - 30):
        c, s = gpu.b.spinner_int_quantize(x[r0:r0 + 30].contiguous(), d, block)
        assert t.equal(codes[r0:r0 + 30], c) and t.equal(scales[r0:r0 + 30], s), r0
    # all of them against the number that they stand for: rotated twice is what went in
    y = gpu.b.spinner_int_dequantize(codes, scales, t.float32, k).double()
    v = x.double()
    if block:
        size = 1
        v = (v * d.double()).view(rows, -1, block)
        while size < block:
            v = v.view(rows, -1, 2, size)
            v = t.stack((v[:, :, 0] + v[:, :, 1], v[:, :, 0] - v[:, :, 1]), 2)
            size *= 2
        v = v.reshape(rows, k) / block ** 0.5
        norm = (x.double() ** 2).view(rows, -1, block).sum(-1).sqrt().amax(-1, keepdim=True)
        off = (np.log2(block) + 3) * 2.0 ** -24 * norm
    else:
        off = 0.0
    s = scales.double()[:, None]
    assert bool(((y - v).abs() <= s * (0.5 + 3e-5) + off + y.abs() * 2.0 ** -24).all())


@pytest.mark.parametrize("k,block", [(70, 0), (512, 256), (4096, 4096), (4100, 0), (20480, 2048)])
def test_rows_to_their_places(gpu, k, block):
    """Codes and scales at their places have the bits of those without, from strided rows and repeated ones too; places outside are passed over."""
    say("int places", k, block)
    t = gpu.torch
    rng = np.random.default_rng(k)
    rows, top = 13, 3
    for name in ("bf16", "f32"):
        x, _ = held(gpu, rng.standard_normal((rows, k + 24)), name)
        d, _ = held(gpu, np.sign(rng.standard_normal(k)))
        d = d if block else None
        p = rng.permutation(rows * top).reshape(rows, top).astype(np.int32)
        for rowsx in (x[:, :k], x[:1, :k].expand(rows, k)):
            codes, scales = gpu.b.spinner_int_quantize(rowsx.contiguous(), d, block)
            c, s = gpu.b.spinner_int_quantize(rowsx, d, block)
            assert t.equal(c, codes) and t.equal(s, scales)
            c, s = gpu.b.spinner_int_quantize(rowsx, d, block, t.from_numpy(p).to(gpu.dev))
            flat = t.from_numpy(p.reshape(-1)).long().to(gpu.dev)
            assert t.equal(c[flat], codes.repeat_interleave(top, 0)) and t.equal(s[flat], scales.repeat_interleave(top))
        q = p.copy()
        q[4, 1], q[5, 2] = -7, rows * top
        c = t.full((rows * top, width(k)), 99, dtype=t.int8, device=gpu.dev)
        s = t.full((rows * top,), 99.0, device=gpu.dev)
        gpu.b.spinner_int_quantize(x[:, :k], d, block, t.from_numpy(q).to(gpu.dev), c, s)
        for at in (p[4, 1], p[5, 2]):
            assert (c[int(at)] == 99).all() and s[int(at)] == 99


def check_products(got, want, name):
    assert np.all(np.abs(got - want) <= np.abs(want) * 1.01 * (HALF_STEP[name] + 3 * 2.0 ** -24) + TINY[name]), np.abs(got - want).max()


def ragged(rng, rows, experts, spare=0):
    ends = np.concatenate((np.sort(rng.integers(0, rows - spare + 1, experts - 1)), [rows - spare]))
    if experts > 3:
        ends[1] = ends[0]
    return np.maximum.accumulate(ends).astype(np.int64)


PRODUCTS = [(1, 16, 1, 1), (1, 4096, 100, 2), (5, 33, 7, 2), (16, 100, 129, 1), (24, 256, 129, 8), (17, 17, 33, 1), (40, 72, 64, 3), (64, 1000, 200, 1), (100, 33, 7, 5),
            (130, 640, 128, 2), (200, 1000, 130, 64), (257, 2048, 256, 1), (500, 100, 60, 65), (700, 1290, 257, 4), (900, 5000, 264, 3), (4100, 700, 1100, 1), (17000, 300, 520, 3), (1500, 2000, 1500, 1), (1300, 300, 2900, 1), (16, 40, 5200, 1), (20, 50, 5111, 2), (7, 24, 17000, 1),
            (70, 1100, 4100, 1), (130, 520, 4500, 2), (300, 72, 4400, 1), (300, 200, 2100, 3), (45, 1500, 6100, 1), (16, 1000, 5000, 1), (20, 700, 5111, 2), (9, 1000, 9000, 1), (64, 1000, 2100, 4),
            (40, 300, 2500, 2), (320, 100, 3300, 4), (1000, 4100, 70, 3)]


@pytest.mark.parametrize("rows,k,n,experts", PRODUCTS)
def test_products(gpu, rows, k, n, experts):
    say("int product", rows, k, n, experts)
    t = gpu.torch
    rng = np.random.default_rng(rows + k + n + experts)
    a = rng.integers(-128, 128, (rows, k))
    w = rng.integers(-128, 128, (experts, n, k))
    a[0], w[0, 0] = -128, -128                               # the largest sum there is
    pad = [(0, 0)] * 2 + [(0, width(k) - k)]
    at = t.from_numpy(np.pad(a, pad[1:]).astype(np.int8)).to(gpu.dev)
    wt = t.from_numpy(np.pad(w, pad).astype(np.int8)).to(gpu.dev)
    sa, sae = held(gpu, np.exp(rng.standard_normal(rows)) / 40)
    sw, swe = held(gpu, np.exp(rng.standard_normal((experts, n))) / 4000)
    every = [ragged(rng, rows, experts), ragged(rng, rows, experts, rows // 4), rng.integers(-5, rows + 5, experts)]
    for ends in every + ([None] if experts == 1 else []):
        e = None if ends is None else t.from_numpy(ends).to(gpu.dev)
        want = ex.int_products(a, sae, w, swe, ends)
        for name in ("f32", "bf16", "f16"):
            check_products(numbers(gpu.b.spinner_int_matmul(at, sa, wt, sw, e, gpu.types[name])), want, name)
    out = t.full((rows, n + 9), 4.0, device=gpu.dev)
    gpu.b.spinner_int_matmul(at, sa, wt, sw, e, t.float32, out=out[:, :n])
    check_products(numbers(out[:, :n]), want, "f32")
    assert (out[:, n:] == 4).all()


def test_deepest_sums(gpu):
    """All codes -128 over the longest rows that are taken: the sum is 2^31 less 2^18."""
    say("int deepest")
    t = gpu.torch
    k = (1 << 17) - 16
    for rows in (3, 70):
        a, w = t.full((rows, k), -128, dtype=t.int8, device=gpu.dev), t.full((40, k), -128, dtype=t.int8, device=gpu.dev)
        y = gpu.b.spinner_int_matmul(a, t.ones(rows, device=gpu.dev), w, t.ones(40, device=gpu.dev), dtype=t.float32)
        assert (y == float(k << 14)).all()


LAYERS = [(1, 4096, 300, 1, 4096), (1, 100, 33, 1, 0), (2, 2048, 64, 1, 256), (8, 512, 200, 1, 512), (3, 1001, 40, 1, 0), (1, 4096, 2100, 2, 1024), (8, 480, 130, 4, 32), (7, 512, 96, 9, 0),
          (37, 1000, 100, 1, 0), (100, 768, 300, 3, 256), (300, 2048, 520, 4, 2048), (1, 64, 33000, 1, 32), (3, 500, 32800, 1, 0)]


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,k,n,experts,block", LAYERS)
def test_layers_are_their_two_calls(gpu, name, rows, k, n, experts, block):
    say("int linear", name, rows, k, n, experts, block)
    t = gpu.torch
    rng = np.random.default_rng(rows + k + n)
    x, _ = held(gpu, rng.standard_normal((rows, k)) * np.where(rng.random(k) < 0.05, 10.0, 1.0), name)
    d, _ = held(gpu, np.sign(rng.standard_normal(k)))
    d = d if block else None
    wc, ws = gpu.b.spinner_int_quantize(held(gpu, rng.standard_normal((experts * n, k)))[0], d, block)
    wc, ws = wc.view(experts, n, -1), ws.view(experts, n)
    ends = t.from_numpy(ragged(rng, rows, experts, rows // 5)).to(gpu.dev)
    codes, scales = gpu.b.spinner_int_quantize(x, d, block)
    y = gpu.b.spinner_int_linear(x, wc, ws, d, block, ends)
    assert t.equal(y, gpu.b.spinner_int_matmul(codes, scales, wc, ws, ends, gpu.types[name]))
    check_products(numbers(y), ex.int_products(whole(codes, k), scales.cpu().numpy(), whole(wc, k), ws.cpu().numpy(), ends.cpu().numpy()), name)
    wide = t.cat((x, x), 1)[:, :k]
    assert t.equal(gpu.b.spinner_int_linear(wide, wc, ws, d, block, ends), y)
    top = 2
    p = rng.permutation(rows * top).reshape(rows, top).astype(np.int32)
    places = t.from_numpy(p).to(gpu.dev)
    ends2 = t.from_numpy(ragged(rng, rows * top, experts, 1)).to(gpu.dev)
    y2 = gpu.b.spinner_int_linear(x, wc, ws, d, block, ends2, places)
    assert t.equal(y2, gpu.b.spinner_int_linear(gpu.b.spinner_dispatch(x, places), wc, ws, d, block, ends2))


def test_no_rows(gpu):
    t, b = gpu.torch, gpu.b
    codes, scales = b.spinner_int_quantize(t.zeros((0, 40), device=gpu.dev))
    assert codes.shape == (0, 48) and scales.shape == (0,) and b.spinner_int_dequantize(codes, scales, k=40).shape == (0, 40)
    w, ws = b.spinner_int_quantize(t.ones((5, 40), device=gpu.dev))
    assert b.spinner_int_matmul(codes, scales, w, ws).shape == b.spinner_int_linear(t.zeros((0, 40), device=gpu.dev), w, ws).shape == (0, 5)
