"""4-bit numbers on the GPU against their 64-bit definitions (oracle/mx4_oracle.py).

Tolerances.  Without a rotation the quantisation is a function of exactly held numbers: equal bytes.  With one, a coordinate v
carries the fp32 rounding of its diagonal product and of log2(block) butterfly stages, each of relative size 2^-24 in norm, so
|error| <= (log2(block) + 3) 2^-24 |run|_2 =: delta, and codes and scales must be those of numbers within delta of the exact
one.  A product of 4-bit numbers is exact; its fp32 sum passes through at most k / 64 + 64 additions, each off by at most
2^-23 of the sum of magnitudes (the matrix pipe may cut where it adds), and is rounded once to the type of the result."""
import sys

import numpy as np
import pytest

from oracle import mx4_oracle as mx

pytestmark = pytest.mark.gpu
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


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


def outliers(rng, rows, k):
    x = rng.standard_normal((rows, k))
    x[:, rng.random(k) < 0.05] *= 10
    return x


def held(g, x, name):
    """x in a type, on the GPU, and the numbers it then holds."""
    t = g.torch.from_numpy(np.ascontiguousarray(x)).to(g.types[name]).to(g.dev)
    return t, t.double().cpu().numpy()


def numbers(t):
    return t.double().cpu().numpy()


def random_packed(rng, rows, k, lo=118, hi=130):
    codes = rng.integers(0, 16, (rows, k)).astype(np.uint8)
    return mx.pack(codes), rng.integers(lo, hi, (rows, k // 32)).astype(np.uint8)


# ---------------------------------------------------------------------------------------------------------- quantise
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,k", [(1, 32), (3, 64), (5, 96), (2, 480), (7, 512), (4, 544), (33, 1024), (1, 4096), (9, 8224), (1000, 160)])
def test_quantise_and_back(gpu, name, rows, k):
    say("quantise", name, rows, k)
    rng = np.random.default_rng(rows * 31 + k)
    x, exact = held(gpu, outliers(rng, rows, k) * np.exp2(rng.integers(-12, 12, (rows, 1))), name)
    codes, scales = gpu.b.spinner_mx_quantize(x)
    want, byte = mx.quantize(exact)
    assert np.array_equal(codes.cpu().numpy(), mx.pack(want))
    assert np.array_equal(scales.cpu().numpy(), byte)
    for out in ("f32", "bf16", "f16"):
        got = gpu.b.spinner_mx_dequantize(codes, scales, gpu.types[out])
        assert got.dtype == gpu.types[out]
        back = gpu.torch.from_numpy(mx.values(mx.pack(want), byte)).to(gpu.types[out])       # one rounding, exact but for fp16's range
        assert np.array_equal(numbers(got), numbers(back), equal_nan=True)


def test_quantise_the_ends_of_the_range(gpu):
    say("quantise: ends of the range")
    rng = np.random.default_rng(3)
    x = np.zeros((40, 64), np.float32)
    x[0, 3], x[1, 40], x[2, 0], x[2, 33] = np.nan, np.inf, -np.inf, 1.0
    x[3] = 2.0 ** -149 * rng.integers(-9, 9, 64)                                  # subnormal numbers
    x[4] = 2.0 ** -126 * rng.standard_normal(64)
    x[5] = 2.0 ** 125 * rng.uniform(-7, 7, 64)
    x[6] = -0.0
    x[7] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, -0.25, 4.0, 7.99, 6.0, 0.0, -0.0, 0.2500001, 0.7499999], 4)
    x[8], x[9] = 8.0, np.nextafter(np.float32(8.0), np.float32(0))
    x[10:] = rng.standard_normal((30, 64)) * np.exp2(rng.integers(-130, 120, (30, 1)))
    x[11, 7] = 3.4e38
    t = gpu.torch.from_numpy(x).to(gpu.dev)
    codes, scales = gpu.b.spinner_mx_quantize(t)
    want, byte = mx.quantize(x.astype(np.float64))
    assert np.array_equal(scales.cpu().numpy(), byte)
    assert np.array_equal(codes.cpu().numpy(), mx.pack(want))
    got, back = numbers(gpu.b.spinner_mx_dequantize(codes, scales)), mx.values(mx.pack(want), byte)
    assert np.array_equal(np.isnan(got), np.isnan(back)) and np.array_equal(got[~np.isnan(got)], back[~np.isnan(back)].astype(np.float32))


def check_rotated(codes, scales, exact, diag, block):
    """Codes and scales are those of numbers within delta of the exact rotation's."""
    v = mx.rotate(exact, diag, block)
    run = np.linalg.norm((exact * (1 if diag is None else diag)).reshape(exact.shape[0], -1, block), axis=-1)
    delta = np.repeat((np.log2(block) + 3) * 2.0 ** -24 * run, block, -1)
    top = np.abs(v).reshape(*v.shape[:-1], -1, 32)
    d32 = delta.reshape(top.shape)
    low, high = mx.scale_bytes(np.maximum(top - d32, 0).max(-1)), mx.scale_bytes((top + d32).max(-1))
    assert np.all((scales >= low) & (scales <= high))
    unit = np.repeat(np.exp2(scales.astype(float) - 127), 32, -1)
    signed = lambda u: np.where(u < 0, -1.0, 1.0) * mx.VALUES[mx.round_to_codes(u) & 7]            # noqa: E731
    got = mx.values(codes, scales) / unit
    assert np.all(got >= signed((v - delta) / unit)) and np.all(got <= signed((v + delta) / unit))


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("block", [32, 64, 128, 256, 512, 1024, 2048, 4096])
def test_rotate_and_quantise(gpu, name, block):
    rng = np.random.default_rng(block)
    for rows, k in ((3, block), (21, 3 * block) if block != 1024 else (21, 5 * block)):
        say("rotate and quantise", name, block, rows, k)
        x, exact = held(gpu, outliers(rng, rows, k), name)
        d = rng.choice([-1.0, 1.0], k).astype(np.float32)
        codes, scales = gpu.b.spinner_mx_quantize(x, gpu.torch.from_numpy(d).to(gpu.dev), block)
        check_rotated(codes.cpu().numpy(), scales.cpu().numpy(), exact, d.astype(np.float64), block)
        codes, scales = gpu.b.spinner_mx_quantize(x, None, block)
        check_rotated(codes.cpu().numpy(), scales.cpu().numpy(), exact, None, block)


def test_rotation_with_an_adaptive_diagonal_and_exact_sums(gpu):
    """Small whole numbers: every sum is exact, so codes and scales are equal."""
    say("rotation, exact sums")
    rng = np.random.default_rng(8)
    for block in (64, 256, 1024, 4096):                    # sqrt(block) is a power of two
        x = rng.integers(-8, 9, (13, 2 * block)).astype(np.float32)
        d = rng.integers(-4, 5, 2 * block).astype(np.float32)
        codes, scales = gpu.b.spinner_mx_quantize(gpu.torch.from_numpy(x).to(gpu.dev), gpu.torch.from_numpy(d).to(gpu.dev), block)
        want, byte = mx.quantize(mx.rotate(x, d, block))
        assert np.array_equal(scales.cpu().numpy(), byte) and np.array_equal(codes.cpu().numpy() & 0x77, mx.pack(want) & 0x77)


def test_no_number_stays_in_its_run(gpu):
    say("NaN and infinity in a rotated run")
    x = np.random.default_rng(2).standard_normal((4, 512)).astype(np.float32)
    x[1, 70], x[2, 300] = np.nan, np.inf
    for block in (0, 128):
        _, scales = gpu.b.spinner_mx_quantize(gpu.torch.from_numpy(x).to(gpu.dev), None, block)
        bad = scales.cpu().numpy() == 255
        want = np.zeros((4, 16), bool)
        if block:
            want[1, 0:4] = want[2, 8:12] = True
        else:
            want[1, 2] = want[2, 9] = True
        assert np.array_equal(bad, want)


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("block", [0, 64, 2048])
def test_rows_any_distance_apart(gpu, name, block):
    say("quantise: strides", name, block)
    t, rng = gpu.torch, np.random.default_rng(4)
    k = 2048
    base, _ = held(gpu, rng.standard_normal((11, 2 * k + 24)), name)
    whole = base[:, :k].contiguous()
    want = gpu.b.spinner_mx_quantize(whole, None, block)
    views = [base[:, :k], base[::2, :k], base[:1, :k].expand(5, k), base.view(-1)[: 11 * (k + 3)].view(11, k + 3)[:, :k]]
    for v in views:
        got = gpu.b.spinner_mx_quantize(v, None, block)
        same = gpu.b.spinner_mx_quantize(v.contiguous(), None, block)
        assert all(t.equal(a, b) for a, b in zip(got, same))
    assert t.equal(gpu.b.spinner_mx_quantize(views[0], None, block)[0], want[0])
    out = t.full((11, k + 5), 7.0, device=gpu.dev, dtype=gpu.types[name])
    gpu.b.spinner_mx_dequantize(*want, dtype=gpu.types[name], out=out[:, :k])
    assert t.equal(out[:, :k], gpu.b.spinner_mx_dequantize(*want, dtype=gpu.types[name])) and bool((out[:, k:] == 7).all())


# ---------------------------------------------------------------------------------------------------------- products
def check_product(got, a, w, out, k):
    want = a @ w.T
    off = np.abs(got - want)
    # one rounding of the result itself, and the sum's error
    bound = np.abs(want) * 1.01 * HALF_STEP[out] + (np.abs(a) @ np.abs(w).T) * (k / 64 + 64) * 2.0 ** -23 + TINY[out]
    assert np.all(off <= bound), float((off / bound).max())


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", [(1, 32, 1), (1, 4096, 1000), (2, 96, 17), (16, 288, 33), (17, 1056, 70), (31, 64, 129), (37, 2048, 257),
                                      (64, 512, 16), (65, 544, 40), (100, 1024, 130), (129, 160, 127), (257, 256, 300), (300, 2080, 515),
                                      (1000, 320, 77), (5, 8192, 64), (700, 4128, 600)])
def test_product(gpu, out, rows, k, n):
    say("product", out, rows, k, n)
    rng = np.random.default_rng(rows + 7 * k + n)
    ac, as_ = random_packed(rng, rows, k, 112, 120)
    wc, ws = random_packed(rng, n, k, 116, 122)
    up = lambda v: gpu.torch.from_numpy(v).to(gpu.dev)                                             # noqa: E731
    got = gpu.b.spinner_mx_matmul(up(ac), up(as_), up(wc), up(ws), dtype=gpu.types[out])
    assert got.dtype == gpu.types[out] and got.shape == (rows, n)
    check_product(numbers(got), mx.values(ac, as_), mx.values(wc, ws), out, k)


def test_product_of_small_whole_numbers_is_exact(gpu):
    say("product, exact")
    rng = np.random.default_rng(12)
    for rows, k, n in ((3, 512, 40), (140, 1056, 200)):
        ac, wc = random_packed(rng, rows, k)[0], random_packed(rng, n, k)[0]
        one = lambda r: np.full((r, k // 32), 128, np.uint8)                                       # noqa: E731
        up = lambda v: gpu.torch.from_numpy(v).to(gpu.dev)                                         # noqa: E731
        got = gpu.b.spinner_mx_matmul(up(ac), up(one(rows)), up(wc), up(one(n)), dtype=gpu.torch.float32)
        assert np.array_equal(numbers(got), mx.values(ac, one(rows)) @ mx.values(wc, one(n)).T)


def ragged(rng, rows, experts, spare=0):
    cut = np.sort(rng.integers(0, rows - spare + 1, experts - 1))
    ends = np.concatenate((cut, [rows - spare]))
    if experts > 3:
        ends[1] = ends[0]                                  # an expert without rows
    return np.maximum.accumulate(ends).astype(np.int64)


GROUPS = [(1, 64, 32, 2), (7, 96, 50, 5), (64, 256, 129, 32), (130, 544, 64, 3), (500, 320, 200, 8), (1030, 256, 70, 16), (90, 64, 40, 63),
          (90, 64, 40, 64), (300, 64, 33, 65), (200, 128, 20, 200), (1200, 288, 260, 4)]


@pytest.mark.parametrize("rows,k,n,experts", GROUPS)
def test_product_by_expert(gpu, rows, k, n, experts):
    say("product by expert", rows, k, n, experts)
    rng = np.random.default_rng(rows + k + n + experts)
    ac, as_ = random_packed(rng, rows, k, 112, 120)
    wc, ws = random_packed(rng, experts * n, k, 116, 122)
    up = lambda v: gpu.torch.from_numpy(v).to(gpu.dev)                                             # noqa: E731
    w = mx.values(wc, ws).reshape(experts, n, k)
    for ends in (ragged(rng, rows, experts), ragged(rng, rows, experts, rows // 5), np.zeros(experts, np.int64),
                 np.full(experts, rows, np.int64), rng.integers(-9, rows + 9, experts)):
        got = numbers(gpu.b.spinner_mx_matmul(up(ac), up(as_), up(wc).view(experts, n, -1), up(ws).view(experts, n, -1), up(ends), gpu.torch.float32))
        last = 0
        for e, (lo, hi) in enumerate(mx.bounds(ends, experts, rows)):
            check_product(got[lo:hi], mx.values(ac, as_)[lo:hi], w[e], "f32", k)
            last = hi
        assert not got[last:].any()


def test_nan_scales_touch_their_own_results_only(gpu):
    say("product, NaN scales")
    rng = np.random.default_rng(6)
    for rows in (5, 90, 200):
        k, n, experts = 320, 140, 3
        ac, as_ = random_packed(rng, rows, k, 112, 120)
        wc, ws = random_packed(rng, experts * n, k, 116, 122)
        ends = np.array([rows // 3, rows // 2, rows - 2])
        as_[1, 4] = as_[rows - 1, 0] = ws[n + 7, 9] = 255                # a row of the first expert, one of none, a column of the second
        up = lambda v: gpu.torch.from_numpy(v).to(gpu.dev)                                         # noqa: E731
        got = numbers(gpu.b.spinner_mx_matmul(up(ac), up(as_), up(wc).view(experts, n, -1), up(ws).view(experts, n, -1), up(ends), gpu.torch.float32))
        want = np.zeros((rows, n), bool)
        want[1] = True
        want[rows // 3:rows // 2, 7] = True
        assert np.array_equal(np.isnan(got), want) and not got[rows - 2:].any()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n,block,experts", [(1, 4096, 200, 4096, 1), (1, 256, 64, 0, 1), (3, 1280, 100, 256, 1), (20, 1024, 65, 32, 4), (37, 2048, 130, 1024, 1),
                                                    (150, 512, 300, 128, 6), (260, 320, 257, 64, 1)])
def test_layer_is_quantise_then_product(gpu, name, rows, k, n, block, experts):
    say("layer", name, rows, k, n, block, experts)
    t, rng = gpu.torch, np.random.default_rng(k + n)
    x, exact = held(gpu, outliers(rng, rows, k), name)
    d = t.from_numpy(rng.choice([-1.0, 1.0], k).astype(np.float32)).to(gpu.dev) if block else None
    w, _ = held(gpu, outliers(rng, experts * n, k), "f32")
    wc, ws = gpu.b.spinner_mx_quantize(w, d, block)
    ends = None
    if experts > 1:
        wc, ws, ends = wc.view(experts, n, -1), ws.view(experts, n, -1), t.from_numpy(ragged(rng, rows, experts, 1)).to(gpu.dev)
    got = gpu.b.spinner_mx_linear(x, wc, ws, d, block, ends)
    ac, as_ = gpu.b.spinner_mx_quantize(x, d, block)
    a, wv = mx.values(ac.cpu().numpy(), as_.cpu().numpy()), mx.values(wc.cpu().numpy(), ws.cpu().numpy()).reshape(experts, n, k)
    for e, (lo, hi) in enumerate(mx.bounds(None if ends is None else ends.cpu().numpy(), experts, rows)):
        check_product(numbers(got)[lo:hi], a[lo:hi], wv[e], name, k)
    # 4 bits with a rotation keep about a tenth of a product of such vectors (16 values, uniform steps within a binade)
    if block >= 256 and experts == 1:
        want = exact @ numbers(w).T
        assert np.linalg.norm(numbers(got) - want) / np.linalg.norm(want) < 0.25
    scratch = t.empty(gpu.b.spinner_mx_linear_workspace_bytes(rows, k), dtype=t.uint8, device=gpu.dev)
    out = t.full((rows, n + 3), 5.0, dtype=x.dtype, device=gpu.dev)
    gpu.b.spinner_mx_linear(x, wc, ws, d, block, ends, out[:, :n], scratch)
    assert t.equal(out[:, :n], got) and bool((out[:, n:] == 5).all())


# ---------------------------------------------------------------------------------------------------------- how it is called
def test_both_ways_of_a_call_and_other_streams(gpu):
    say("native and long way, streams")
    t, b, rng = gpu.torch, gpu.b, np.random.default_rng(1)
    x, _ = held(gpu, rng.standard_normal((40, 512)), "bf16")
    w, _ = held(gpu, rng.standard_normal((3 * 48, 512)), "f32")
    d = t.ones(512, device=gpu.dev)
    ends = t.tensor([10, 10, 39], device=gpu.dev)
    wc, ws = (v.view(3, 48, -1) for v in b.spinner_mx_quantize(w, d, 256))
    ac, as_ = b.spinner_mx_quantize(x, d, 256)
    calls = [lambda **k: b.spinner_mx_quantize(x, d, 256, **k), lambda **k: b.spinner_mx_dequantize(ac, as_, t.float16, **k),
             lambda **k: b.spinner_mx_matmul(ac, as_, wc, ws, ends, t.float32, **k), lambda **k: b.spinner_mx_linear(x, wc, ws, d, 256, ends, **k)]
    side = t.cuda.Stream()
    for call in calls:
        first = call()
        side.wait_stream(t.cuda.current_stream())
        other = call(stream=side)
        side.synchronize()
        for p, q in zip(first, other) if isinstance(first, tuple) else [(first, other)]:
            assert t.equal(p, q)


def test_captured_graph_gives_the_eager_bits(gpu):
    say("graph capture")
    t, b, rng = gpu.torch, gpu.b, np.random.default_rng(9)
    w, _ = held(gpu, rng.standard_normal((2 * 80, 1024)), "f32")
    d = t.from_numpy(rng.choice([-1.0, 1.0], 1024).astype(np.float32)).to(gpu.dev)
    wc, ws = (v.view(2, 80, -1) for v in b.spinner_mx_quantize(w, d, 1024))
    ends = t.tensor([30, 70], device=gpu.dev)
    x, _ = held(gpu, rng.standard_normal((75, 1024)), "bf16")
    out = t.zeros((75, 80), dtype=x.dtype, device=gpu.dev)
    scratch = t.empty(b.spinner_mx_linear_workspace_bytes(75, 1024), dtype=t.uint8, device=gpu.dev)
    call = lambda: b.spinner_mx_linear(x, wc, ws, d, 1024, ends, out, scratch)                     # noqa: E731
    call()
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        call()
    for k in range(4):
        x.copy_(t.from_numpy(rng.standard_normal((75, 1024))).to(x.dtype))
        ends.copy_(t.tensor([20 + 10 * k, 75 - k]))
        out.zero_()
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out, b.spinner_mx_linear(x, wc, ws, d, 1024, ends))


def test_places_beyond_32_bits(gpu):
    say("offsets beyond 32 bits")
    t, b = gpu.torch, gpu.b
    rows, k, n = (1 << 21) + 77, 2080, 1040                # 4.4e9 numbers in, 2.2e9 out
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(1)
    part = t.randn((1 << 14, k), generator=gen, device=gpu.dev, dtype=t.float32).to(t.bfloat16)
    x = t.empty((rows, k), dtype=t.bfloat16, device=gpu.dev)
    for r in range(0, rows, 1 << 14):
        x[r:r + (1 << 14)] = part[: rows - r]
    wc, ws = b.spinner_mx_quantize(t.randn((n, k), generator=gen, device=gpu.dev), None, 32)
    y = b.spinner_mx_linear(x, wc, ws, None, 32)
    at = (rows >> 14) << 14
    assert t.equal(y[at:], b.spinner_mx_linear(x[at:].clone(), wc, ws, None, 32)) or \
        t.allclose(y[at:].float(), b.spinner_mx_linear(x[at:].clone(), wc, ws, None, 32).float(), rtol=2.0 ** -7, atol=1e-3)
    assert t.equal(y[:256], y[1 << 14:(1 << 14) + 256]) and t.equal(y[at - (1 << 14):at - (1 << 14) + 256], y[:256])
    codes, scales = b.spinner_mx_quantize(x, None, 32)
    assert t.equal(codes[at:], codes[: rows - at]) and t.equal(scales[at:], scales[: rows - at])
    back = b.spinner_mx_dequantize(codes, scales, t.bfloat16)
    assert t.equal(back[at:], back[: rows - at])


def test_refusals(gpu):
    say("refusals")
    t, b = gpu.torch, gpu.b
    x = t.zeros((4, 128), device=gpu.dev)
    codes, scales = b.spinner_mx_quantize(x)
    w3, s3 = codes.view(2, 2, 64), scales.view(2, 2, 4)
    ends = t.tensor([1, 4], device=gpu.dev)

    def status(code, call):
        with pytest.raises(b.SpinnerError) as e:
            call()
        assert e.value.status == code

    status(b.SPINNER_ERR_BAD_SHAPE, lambda: b.spinner_mx_quantize(x[:, :100]))
    status(b.SPINNER_ERR_BAD_SHAPE, lambda: b.spinner_mx_quantize(x, None, 16))
    status(b.SPINNER_ERR_BAD_SHAPE, lambda: b.spinner_mx_quantize(x, None, 96))
    status(b.SPINNER_ERR_BAD_SHAPE, lambda: b.spinner_mx_quantize(x, None, 256))
    status(b.SPINNER_ERR_BAD_SHAPE, lambda: b.spinner_mx_quantize(x, t.ones(128, device=gpu.dev), 0))
    status(b.SPINNER_ERR_BAD_TYPE, lambda: b.spinner_mx_quantize(x.double()))
    status(b.SPINNER_ERR_BAD_TYPE, lambda: b.spinner_mx_dequantize(codes, scales, t.int32))
    status(b.SPINNER_ERR_ALIGNMENT, lambda: b.spinner_mx_quantize(t.zeros(4 * 128 + 1, device=gpu.dev)[1:].view(4, 128)))
    for bad in (lambda: b.spinner_mx_quantize(x.cpu()), lambda: b.spinner_mx_quantize(x.t()), lambda: b.spinner_mx_quantize(x[0]),
                lambda: b.spinner_mx_quantize(x, t.ones(64, device=gpu.dev), 64), lambda: b.spinner_mx_quantize(x, codes=codes[:2]),
                lambda: b.spinner_mx_dequantize(codes, scales[:2]), lambda: b.spinner_mx_dequantize(codes, scales, out=x.half()),
                lambda: b.spinner_mx_matmul(codes, scales, codes[:, :32].contiguous(), scales),
                lambda: b.spinner_mx_matmul(codes, scales, w3, s3), lambda: b.spinner_mx_matmul(codes, scales, w3, s3, ends[:1]),
                lambda: b.spinner_mx_matmul(codes, scales, w3, s3, ends.int()), lambda: b.spinner_mx_matmul(codes, scales, w3, s3, ends.cpu()),
                lambda: b.spinner_mx_linear(x.half(), w3, s3, ends=ends, out=x), lambda: b.spinner_mx_linear(x[:, :64], w3, s3, ends=ends),
                lambda: b.spinner_mx_linear(x, w3, s3, ends=ends, workspace=codes[:1, :8].contiguous()),
                lambda: b.spinner_mx_linear(x, w3, s3, ends=ends, out=t.zeros((1, 2), device=gpu.dev).expand(4, 2))):
        with pytest.raises(ValueError):
            bad()
    empty = b.spinner_mx_linear(x[:0], w3, s3, ends=ends)
    assert empty.shape == (0, 2)
