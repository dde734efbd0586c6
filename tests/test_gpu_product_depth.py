"""Every form of the products through many chunks of depth (product_forms.py), against 64-bit products; and the same bits each time.

Tolerances as in test_gpu_product_forms.py: (depth / 16 + 16) 2^-23 of the sum of magnitudes for 16-bit operands (weight gradients, with their shares,
depth / 16 + 32), (k / 64 + 64) 2^-23 for 4-bit ones, and one rounding of the result."""
import sys

import numpy as np
import pytest

import product_forms as forms
from oracle import mx4_oracle as mx
from test_gpu_product_forms import check, ragged

pytestmark = pytest.mark.gpu


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


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("rows,experts,k,n", forms.SIXTEEN)
def test_sixteen_bits(gpu, name, rows, experts, k, n):
    say("depth", name, rows, experts, k, n, [forms.plan(d, False, rows, experts, k, n) for d in (0, 1, 2)])
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(rows + k + n)
    x, dy, w = (t.randn(s, generator=gen, device=gpu.dev).to(gpu.types[name]) for s in ((rows, k), (rows, n), (experts, n, k)))
    ends = None if experts == 1 else ragged(np.random.default_rng(rows), rows, experts, 3)
    e = None if ends is None else t.from_numpy(ends).to(gpu.dev)
    if experts == 1:
        w = w[0]
    calls = [lambda: b.spinner_grouped_matmul(x, w, e), lambda: b.spinner_grouped_matmul_dx(dy, w, e), lambda: b.spinner_grouped_matmul_dw(dy, x, e, gpu.types[name]),
             lambda: b.spinner_grouped_matmul_dw(dy, x, e)]
    y, dx, dw16, dw = (c() for c in calls)
    for i, (lo, hi) in enumerate(mx.bounds(ends, experts, rows)):
        xe, dye, we = x[lo:hi].double(), dy[lo:hi].double(), (w if experts == 1 else w[i]).double()
        check(y[lo:hi], xe @ we.T, xe.abs() @ we.abs().T, (k / 16 + 16) * 2.0 ** -23, name)
        check(dx[lo:hi], dye @ we, dye.abs() @ we.abs(), (n / 16 + 16) * 2.0 ** -23, name)
        want, size = dye.T @ xe, dye.abs().T @ xe.abs()
        for got, out in ((dw16, name), (dw, "f32")):
            check(got if experts == 1 else got[i], want, size, ((hi - lo) / 16 + 32) * 2.0 ** -23, out)
    for first, call in zip((y, dx, dw16, dw), calls):
        assert t.equal(call(), first)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,experts,k,n", forms.FOUR)
def test_four_bits(gpu, out, rows, experts, k, n):
    say("depth, 4 bits", out, rows, experts, k, n, forms.plan(0, True, rows, experts, k, n))
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(rows + k)
    codes = lambda r: t.randint(0, 256, (r, k // 2), generator=gen, device=gpu.dev, dtype=t.uint8)          # noqa: E731
    scales = lambda r: t.randint(112, 122, (r, k // 32), generator=gen, device=gpu.dev, dtype=t.uint8)      # noqa: E731
    ac, as_, wc, ws = codes(rows), scales(rows), codes(experts * n), scales(experts * n)
    ends = ragged(np.random.default_rng(rows), rows, experts, 5)
    call = lambda: b.spinner_mx_matmul(ac, as_, wc.view(experts, n, -1), ws.view(experts, n, -1), t.from_numpy(ends).to(gpu.dev), gpu.types[out])          # noqa: E731
    y = call()
    a, w = (t.from_numpy(mx.values(c.cpu().numpy(), s.cpu().numpy())).to(gpu.dev) for c, s in ((ac, as_), (wc, ws)))
    w = w.view(experts, n, k)
    assert not bool(y[ends[-1]:].any())
    for i, (lo, hi) in enumerate(mx.bounds(ends, experts, rows)):
        check(y[lo:hi], a[lo:hi] @ w[i].T, a[lo:hi].abs() @ w[i].abs().T, (k / 64 + 64) * 2.0 ** -23, out)
    assert t.equal(call(), y)


def test_a_prompt_gives_the_same_bits_each_time(gpu):
    """Quantisation of runs of 512 (a factor that fp32 rounds) and the largest 4-bit tiles: rows that repeat give equal results, and so does every pass."""
    say("a prompt, time after time")
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(5)
    rows, k, n = 8192, 4096, 4096
    part = t.randn((1024, k), generator=gen, device=gpu.dev).bfloat16()
    x = part.repeat(rows // 1024, 1)
    d = t.randint(0, 2, (k,), generator=gen, device=gpu.dev).float() * 2 - 1
    wc, ws = b.spinner_mx_quantize(t.randn((n, k), generator=gen, device=gpu.dev), d, 512)
    first = b.spinner_mx_linear(x, wc, ws, d, 512)
    for _ in range(12):
        left = t.full((rows, n), float("nan"), device=gpu.dev)           # what is not written would show
        del left
        assert t.equal(b.spinner_mx_linear(x, wc, ws, d, 512), first)
    assert t.equal(first.view(8, 1024, n), first[:1024].expand(8, 1024, n))
    # and what the two calls give that it stands for
    assert t.equal(b.spinner_mx_matmul(*b.spinner_mx_quantize(x, d, 512), wc, ws), first)


# few rows a group: 16, 32 and 64 rows of weights a workgroup, by how many there are; sums of several runs a wave, with and without a rest
@pytest.mark.parametrize("rows,experts,k,n", [(16, 1, 8736, 100), (9, 1, 6656, 16390), (3, 1, 1056, 65550), (40, 32, 2592, 700), (64, 32, 4384, 2100), (300, 64, 544, 1030)])
def test_few_rows_in_4_bits(gpu, rows, experts, k, n):
    assert forms.plan(0, True, rows, experts, k, n)[0] == "few rows"
    test_four_bits(gpu, "f32", rows, experts, k, n)
    test_four_bits(gpu, "bf16", rows, experts, k, n)


@pytest.mark.parametrize("rows,experts,k,n", [(16, 1, 4104, 100), (9, 1, 3333, 1030), (5, 1, 2056, 16390), (40, 32, 1667, 515), (64, 32, 2048, 1024)])
def test_few_rows_in_16_bits(gpu, rows, experts, k, n):
    assert forms.plan(0, False, rows, experts, k, n)[0] == "few rows"
    test_sixteen_bits(gpu, "bf16", rows, experts, k, n)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,experts,k,n,block", [(1, 1, 4096, 65550, 4096), (1, 1, 3552, 65600, 32), (2, 1, 1984, 65537, 64), (8, 8, 512, 8200, 512), (7, 40, 480, 2000, 0)])
def test_layers_of_few_rows_with_many_columns(gpu, name, rows, experts, k, n, block):
    """The form that quantises for itself with 32 rows of weights a wave: the bits of two calls, which are checked against the 64-bit definitions above."""
    say("few rows, many columns", name, rows, experts, k, n, block)
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(rows + k)
    x = t.randn((rows, k), generator=gen, device=gpu.dev).to(gpu.types[name])
    d = t.randint(0, 2, (k,), generator=gen, device=gpu.dev).float() * 2 - 1 if block else None
    wc, ws = b.spinner_mx_quantize(t.randn((experts * n, k), generator=gen, device=gpu.dev), d, block)
    wc, ws = wc.view(experts, n, -1), ws.view(experts, n, -1)
    ends = t.from_numpy(ragged(np.random.default_rng(rows), rows, experts, 0)).to(gpu.dev)
    got = b.spinner_mx_linear(x, wc, ws, d, block, ends)
    ac, as_ = b.spinner_mx_quantize(x, d, block)
    assert t.equal(got, b.spinner_mx_matmul(ac, as_, wc, ws, ends, gpu.types[name]))
    a, w = (t.from_numpy(mx.values(c.cpu().numpy(), s.cpu().numpy())).to(gpu.dev) for c, s in ((ac, as_), (wc.view(experts * n, -1), ws.view(experts * n, -1))))
    w = w.view(experts, n, k)
    for i, (lo, hi) in enumerate(mx.bounds(ends.cpu().numpy(), experts, rows)):
        check(got[lo:hi], a[lo:hi] @ w[i].T, a[lo:hi].abs() @ w[i].abs().T, (k / 64 + 64) * 2.0 ** -23, name)


@pytest.mark.parametrize("rows,experts,k,n", [(3, 1, 1056, 65), (19, 1, 2656, 37), (57, 3, 2784, 32), (113, 3, 1152, 5237), (2050, 1, 1056, 4104), (300, 64, 544, 1030)])
def test_scales_of_any_alignment(gpu, rows, experts, k, n):
    """Scales that start anywhere, at the beginning and at the end of their memory: the bits of aligned ones, from every form."""
    say("scales of any alignment", rows, experts, k, n, forms.plan(0, True, rows, experts, k, n))
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(rows + n)
    codes = lambda r: t.randint(0, 256, (r, k // 2), generator=gen, device=gpu.dev, dtype=t.uint8)          # noqa: E731
    scales = lambda r: t.randint(112, 122, (r, k // 32), generator=gen, device=gpu.dev, dtype=t.uint8)      # noqa: E731

    def moved(s, by):
        flat = t.full((s.numel() + by,), 255, device=gpu.dev, dtype=t.uint8)
        flat[by:] = s.flatten()
        return flat[by:].view(s.shape)

    ac, as_, wc, ws = codes(rows), scales(rows), codes(experts * n).view(experts, n, -1), scales(experts * n).view(experts, n, -1)
    ends = t.from_numpy(ragged(np.random.default_rng(rows), rows, experts, 1)).to(gpu.dev)
    want = b.spinner_mx_matmul(ac, as_, wc, ws, ends, t.float32)
    back = b.spinner_mx_dequantize(ac, as_)
    x = t.randn((rows, k), generator=gen, device=gpu.dev).bfloat16()
    quantised = b.spinner_mx_quantize(x, None, 32)
    for by in (1, 3, 8, 13):
        assert t.equal(b.spinner_mx_matmul(ac, moved(as_, by), wc, moved(ws, 16 - by), ends, t.float32), want)
        assert t.equal(b.spinner_mx_dequantize(ac, moved(as_, by)), back)
        got = b.spinner_mx_quantize(x, None, 32, scales=moved(as_, by))
        assert t.equal(got[0], quantised[0]) and t.equal(got[1], quantised[1])
        assert t.equal(b.spinner_mx_linear(x, wc, moved(ws, by), None, 32, ends), b.spinner_mx_linear(x, wc, ws, None, 32, ends))
