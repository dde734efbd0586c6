"""The products and quantisation at sizes that take more workgroups than one grid holds (2^32 threads)."""
import sys

import numpy as np
import pytest

from oracle import mx4_oracle as mx

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
    yield g
    torch.cuda.empty_cache()


def say(*a):
    print("\n[gpu-case]", *a, file=sys.stderr, flush=True)


def bytes_of(g, rows, width, lo, hi, seed):
    """[rows][width] random bytes, the same 2^16 rows time after time but for the first and the last few, which are their own."""
    t = g.torch
    gen = t.Generator(device=g.dev)
    gen.manual_seed(seed)
    part = t.randint(lo, hi, (1 << 16, width), generator=gen, device=g.dev, dtype=t.uint8)
    out = t.empty((rows, width), dtype=t.uint8, device=g.dev)
    for r in range(0, rows, 1 << 16):
        out[r:r + (1 << 16)] = part[: rows - r]
    for at in (0, rows - 40):
        out[at:at + 40] = t.randint(lo, hi, (40, width), generator=gen, device=g.dev, dtype=t.uint8)
    return out


@pytest.mark.parametrize("name,k,rows", [("float32", 4096, (1 << 22) + 45), ("bfloat16", 8192, (1 << 22) + 45)])
def test_back_from_4_bits_beyond_one_grid(gpu, name, k, rows):
    """2^34 fp32 numbers and more are 2^32 threads of four, 2^35 of 16 bits as many of eight."""
    say("dequantise beyond one grid", name, rows, k)
    t, b = gpu.torch, gpu.b
    t.cuda.empty_cache()
    codes, scales = bytes_of(gpu, rows, k // 2, 0, 256, 1), bytes_of(gpu, rows, k // 32, 100, 140, 2)
    out = b.spinner_mx_dequantize(codes, scales, getattr(t, name))
    half = 1 << 21                                         # numbers of the first half of 2^31 threads: 2^33, of the second and of what is left
    for at in (0, 77777, half - 3, half, (1 << 22) - 9, 1 << 22, rows - 40):
        some = slice(at, min(at + 8, rows))
        want = t.from_numpy(mx.values(codes[some].cpu().numpy(), scales[some].cpu().numpy())).to(getattr(t, name))
        assert t.equal(out[some].cpu(), want), at
    # all of it, 2^16 rows at a time
    for r in range(1 << 16, rows - 40, 1 << 16):
        upto = min(r + (1 << 16), rows - 40)
        assert t.equal(out[r + 40:upto], out[(1 << 16) + 40:(1 << 16) + upto - r])
    assert bool((out[1 << 16:(1 << 16) + 300] != 0).any())


def test_few_results_of_many_rows(gpu):
    """Weights of fewer than sixteen scales: sixteen rows a workgroup, 2^24 workgroups and more."""
    rows, k, n = (1 << 28) + 37, 32, 8
    say("few results of many rows", rows, k, n)
    t, b = gpu.torch, gpu.b
    t.cuda.empty_cache()
    ac, as_ = bytes_of(gpu, rows, k // 2, 0, 256, 3), bytes_of(gpu, rows, 1, 120, 130, 4)
    wc, ws = bytes_of(gpu, 50, k // 2, 0, 256, 5)[:n].contiguous(), bytes_of(gpu, 50, 1, 120, 130, 6)[:n].contiguous()
    out = b.spinner_mx_matmul(ac, as_, wc, ws, dtype=t.float32)
    w = mx.values(wc.cpu().numpy(), ws.cpu().numpy())
    for at in (0, 12345678, 16 * ((1 << 23) - 8) - 5, 16 * ((1 << 23) - 8), 16 * (1 << 24) - 3, rows - 20):
        some = slice(at, min(at + 20, rows))
        a = mx.values(ac[some].cpu().numpy(), as_[some].cpu().numpy())
        # products of 4-bit numbers within 2^20 of one another: exact in fp32 sums of 32
        assert np.array_equal(out[some].cpu().numpy(), (a @ w.T).astype(np.float32)), at
    for r in range(1 << 17, rows - 40, 1 << 24):
        upto = min(r + (1 << 16), rows - 40)
        assert t.equal(out[r + 40:upto], out[(1 << 16) + 40:(1 << 16) + upto - r])


def test_weight_gradients_of_many_columns(gpu):
    """1024 experts by 2^22 + 8 numbers a row: more tiles than one grid holds, all but three of them zeros."""
    rows, k, experts = 40, (1 << 22) + 8, 1024
    say("weight gradients of many columns", rows, k, experts)
    t, b = gpu.torch, gpu.b
    t.cuda.empty_cache()
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(7)
    dy = t.randint(-8, 9, (rows, 1), generator=gen, device=gpu.dev).bfloat16()
    x = t.randint(-8, 9, (rows, k), generator=gen, device=gpu.dev).bfloat16()
    ends = t.full((experts,), 30, dtype=t.int64, device=gpu.dev)
    ends[0], ends[1:600], ends[1023] = 11, 11, 39
    dw = b.spinner_grouped_matmul_dw(dy, x, ends, t.bfloat16)
    used = {0: (0, 11), 600: (11, 30), 1023: (30, 39)}
    for e in range(experts):
        if e not in used:
            assert not bool(dw[e].any()), e
    for e, (lo, hi) in used.items():                       # small whole numbers: sums are exact before the one rounding
        assert t.equal(dw[e, 0], (dy[lo:hi].float() * x[lo:hi].float()).sum(0).bfloat16())


def test_layers_beyond_32_bits_give_the_bits_of_their_parts(gpu):
    """4.4e9 numbers in, 2.2e9 out: the same rows time after time give the same results wherever they lie, and those of the 64-bit definition."""
    rows, k, n = (1 << 21) + 77, 2080, 1040
    say("a layer beyond 32 bits", rows, k, n)
    t, b = gpu.torch, gpu.b
    t.cuda.empty_cache()
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(1)
    part = t.randn((1 << 14, k), generator=gen, device=gpu.dev).bfloat16()
    x = t.empty((rows, k), dtype=t.bfloat16, device=gpu.dev)
    for r in range(0, rows, 1 << 14):
        x[r:r + (1 << 14)] = part[: rows - r]
    wc, ws = b.spinner_mx_quantize(t.randn((n, k), generator=gen, device=gpu.dev), None, 32)
    y = b.spinner_mx_linear(x, wc, ws, None, 32)
    for r in range(1 << 14, rows, 1 << 14):
        assert t.equal(y[r:r + (1 << 14)], y[: min(1 << 14, rows - r)]), r
    ac, as_ = b.spinner_mx_quantize(part[:200], None, 32)
    a, w = (mx.values(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((ac, as_), (wc, ws)))
    want, size = a @ w.T, np.abs(a) @ np.abs(w).T
    # one rounding to bf16, (k / 64 + 64) additions off by at most 2^-23 of the sum of magnitudes
    for at in (0, (rows >> 14) << 14):
        upto = min(200, rows - at)
        off = np.abs(y[at:at + upto].double().cpu().numpy() - want[:upto])
        assert np.all(off <= np.abs(want[:upto]) * 1.01 * 2.0 ** -8 + size[:upto] * (k / 64 + 64) * 2.0 ** -23)
