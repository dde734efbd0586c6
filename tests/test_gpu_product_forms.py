"""The products at sizes that take each form of the kernels (tiles of 256, 128 and 64, four chunks in LDS, sums in shares), whole
pieces of rows and others, against 64-bit products; and that a layer trained in 16 bits can be served from 4-bit weights.

Tolerances as in test_gpu_grouped.py and test_gpu_mx.py: (depth / 16 + 16) 2^-23 of the sum of magnitudes for 16-bit operands (one more
addition a share), (k / 64 + 64) 2^-23 for 4-bit ones, and one rounding of the result."""
import os
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


def ragged(rng, rows, experts, spare):
    ends = np.concatenate((np.sort(rng.integers(0, rows - spare + 1, experts - 1)), [rows - spare]))
    return ends.astype(np.int64)


def check(got, want, size, depth, out):
    off = (got.double() - want).abs()
    bound = want.abs() * (1.01 * HALF_STEP[out]) + size * depth + TINY[out]
    assert bool((off <= bound).all()), float((off / bound).max())


SIZES = [(20000, 40, 136, 3), (20000, 136, 40, 1), (2050, 40, 1032, 3), (2050, 1032, 40, 3), (2050, 40, 4104, 3), (2050, 4104, 40, 1), (70, 4104, 264, 3),
         (70, 4104, 136, 3), (70, 2056, 2056, 3), (2050, 40, 40, 1), (4100, 264, 40, 3), (8200, 1032, 520, 1), (20000, 2056, 136, 3), (600, 520, 1032, 1)]


@pytest.mark.parametrize("off", [0, 3])
@pytest.mark.parametrize("rows,k,n,experts", SIZES)
def test_sixteen_bits(gpu, rows, k, n, experts, off):
    k, n = k + off, n + (1 if off else 0)
    name = "bf16" if (rows + off) % 3 else "f16"
    say("forms", name, rows, k, n, experts)
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(rows + k)
    x, dy, w = (t.randn(s, generator=gen, device=gpu.dev).to(gpu.types[name]) for s in ((rows, k), (rows, n), (experts, n, k)))
    ends = ragged(np.random.default_rng(rows), rows, experts, 5)
    e = t.from_numpy(ends).to(gpu.dev)
    y, dx = b.spinner_grouped_matmul(x, w, e), b.spinner_grouped_matmul_dx(dy, w, e)
    dws = {out: b.spinner_grouped_matmul_dw(dy, x, e, gpu.types[out]) for out in ("f32", name)}
    assert not bool(y[ends[-1]:].any()) and not bool(dx[ends[-1]:].any())
    for i, (lo, hi) in enumerate(mx.bounds(ends, experts, rows)):
        xe, dye, we = x[lo:hi].double(), dy[lo:hi].double(), w[i].double()
        check(y[lo:hi], xe @ we.T, xe.abs() @ we.abs().T, (k / 16 + 16) * 2.0 ** -23, name)
        check(dx[lo:hi], dye @ we, dye.abs() @ we.abs(), (n / 16 + 16) * 2.0 ** -23, name)
        for out, dw in dws.items():
            check(dw[i], dye.T @ xe, dye.abs().T @ xe.abs(), ((hi - lo) / 16 + 32) * 2.0 ** -23, out)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n,experts", [(70, 8224, 40, 1), (70, 16416, 140, 2), (2050, 64, 4104, 3), (1100, 4128, 2051, 1), (3000, 544, 2300, 4), (90, 8192, 333, 1),
                                              (200, 7968, 130, 1), (300, 1120, 515, 2)])
def test_four_bits(gpu, rows, k, n, experts, out):
    say("forms, 4 bits", out, rows, k, n, experts)
    t, b = gpu.torch, gpu.b
    gen = t.Generator(device=gpu.dev)
    gen.manual_seed(rows + k)
    codes = lambda r: t.randint(0, 256, (r, k // 2), generator=gen, device=gpu.dev, dtype=t.uint8)          # noqa: E731
    scales = lambda r: t.randint(112, 124, (r, k // 32), generator=gen, device=gpu.dev, dtype=t.uint8)      # noqa: E731
    ac, as_, wc, ws = codes(rows), scales(rows), codes(experts * n), scales(experts * n)
    ends = ragged(np.random.default_rng(rows), rows, experts, 7)
    y = b.spinner_mx_matmul(ac, as_, wc.view(experts, n, -1), ws.view(experts, n, -1), t.from_numpy(ends).to(gpu.dev), gpu.types[out])
    a, w = (t.from_numpy(mx.values(c.cpu().numpy(), s.cpu().numpy())).to(gpu.dev) for c, s in ((ac, as_), (wc, ws)))
    w = w.view(experts, n, k)
    assert not bool(y[ends[-1]:].any())
    for i, (lo, hi) in enumerate(mx.bounds(ends, experts, rows)):
        check(y[lo:hi], a[lo:hi] @ w[i].T, a[lo:hi].abs() @ w[i].abs().T, (k / 64 + 64) * 2.0 ** -23, out)


def test_shares_of_a_sum_need_their_workspace(gpu):
    say("forms, workspace")
    t, b = gpu.torch, gpu.b
    rows, n, k = 4100, 40, 264
    need = b.spinner_grouped_matmul_dw_workspace_bytes(rows, n, k, 1)
    assert need > 0 and b.spinner_grouped_matmul_dw_workspace_bytes(16, n, k, 1) == 0 and b.spinner_grouped_matmul_dw_workspace_bytes(-1, n, k, 1) == 0
    dy, x = t.randn((rows, n), device=gpu.dev).bfloat16(), t.randn((rows, k), device=gpu.dev).bfloat16()
    want = b.spinner_grouped_matmul_dw(dy, x)
    scratch = t.full((need,), 255, dtype=t.uint8, device=gpu.dev)             # NaN: what is not written shows
    assert t.equal(b.spinner_grouped_matmul_dw(dy, x, workspace=scratch), want)
    with pytest.raises(ValueError):
        b.spinner_grouped_matmul_dw(dy, x, workspace=scratch[:-1])
    rc = b.lib.spinner_grouped_matmul_dw(dy.data_ptr(), x.data_ptr(), 1, rows, n, k, n, k, 1, None, want.data_ptr(), 0, None, None)
    assert rc == b.SPINNER_ERR_WORKSPACE


def test_example_trains_and_serves(gpu):
    say("example")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import expert_layer

    first, last, served, direct = expert_layer.main(rows=2048, n=1024, width=256, experts=8, steps=30, quiet=True)
    assert last < 0.5 * first                                 # the layer learns
    assert served < 2 * last and served < direct              # 4 bits with a rotation serve it, better than without


def test_usual_calls_are_served_natively(gpu):
    """The native part answers the usual calls itself, and hands on what is out of the ordinary (None)."""
    say("native part of the binding")
    t, b = gpu.torch, gpu.b
    native = b._native_products
    x, d, w = t.randn((6, 128), device=gpu.dev), t.ones(128, device=gpu.dev), t.randn((10, 128), device=gpu.dev)
    codes, scales = native.mx_quantize(x, d, 64, None, None, None)
    wc, ws = native.mx_quantize(w, d, 64, None, None, None)
    h, hw, dy = x.bfloat16(), w.bfloat16(), t.randn((6, 10), device=gpu.dev).bfloat16()
    served = [native.mx_dequantize(codes, scales, t.float32, None, None), native.mx_matmul(codes, scales, wc, ws, None, t.float16, None, None),
              native.mx_linear(h, wc, ws, d, 64, None, None, None, None), native.grouped_matmul(h, hw, None, None, None),
              native.grouped_matmul_dx(dy, hw, None, None, None), native.grouped_matmul_dw(dy, h, None, t.float32, None, None, None)]
    assert all(r is not None for r in served)
    side = t.cuda.current_stream()
    handed_on = [native.mx_quantize(x, d, 64, None, None, side), native.mx_quantize(x[:, :64], None, 0, None, None, None), native.mx_quantize(x.cpu(), None, 0, None, None, None),
                 native.mx_quantize(x, d, 48, None, None, None), native.mx_linear(x.double(), wc, ws, d, 64, None, None, None, None),
                 native.grouped_matmul(h, hw.half(), None, None, None), native.grouped_matmul(x, w, None, None, None), native.grouped_matmul(dy, hw, None, None, None)]
    assert all(r is None for r in handed_on)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n,block,experts", [(1, 32, 1, 32, 1), (1, 32, 17, 0, 1), (1, 480, 33, 32, 1), (1, 544, 31, 0, 1), (1, 1536, 70, 512, 1), (1, 2048, 4100, 1024, 1), (1, 4096, 65, 2048, 1),
                                                    (1, 4096, 129, 4096, 1), (1, 3840, 48, 256, 1), (1, 4128, 48, 32, 1), (2, 2048, 100, 2048, 1), (2, 1984, 40, 64, 1), (3, 1024, 200, 512, 1),
                                                    (4, 1024, 31, 1024, 1), (8, 512, 64, 128, 1), (8, 96, 64, 0, 1), (9, 512, 64, 512, 1), (2, 1024, 40, 1024, 5), (5, 480, 50, 32, 3), (1, 2048, 33, 1024, 64)])
def test_layers_of_few_rows_are_quantise_then_product(gpu, name, rows, k, n, block, experts):
    """A row or a few through a layer, where the product's workgroups quantise for themselves (sizes on both sides of that): the same bits as in two calls."""
    say("few rows in one launch", name, rows, k, n, block, experts)
    t, rng = gpu.torch, np.random.default_rng(rows + k + n)
    x = t.from_numpy((rng.standard_normal((rows, k)) * np.where(rng.random(k) < 0.05, 20.0, 1.0)).astype(np.float32)).to(gpu.dev).to(gpu.types[name])
    if rows > 1:
        x[1, k // 2] = float("nan")          # its 32, or its run; all of its row's results
    d = t.from_numpy(rng.standard_normal(k).astype(np.float32)).to(gpu.dev) if block else None
    wc, ws = gpu.b.spinner_mx_quantize(t.from_numpy(rng.standard_normal((experts * n, k)).astype(np.float32)).to(gpu.dev), d, block)
    ends = None
    if experts > 1:
        wc, ws, ends = wc.view(experts, n, -1), ws.view(experts, n, -1), t.from_numpy(ragged(rng, rows, experts, 1 if rows > 2 else 0)).to(gpu.dev)
    got = gpu.b.spinner_mx_linear(x, wc, ws, d, block, ends)
    ac, as_ = gpu.b.spinner_mx_quantize(x, d, block)
    want = gpu.b.spinner_mx_matmul(ac, as_, wc, ws, ends, x.dtype)
    assert t.equal(got.nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
    a, w = mx.values(ac.cpu().numpy(), as_.cpu().numpy()), mx.values(wc.cpu().numpy(), ws.cpu().numpy()).reshape(experts, n, k)
    for e, (lo, hi) in enumerate(mx.bounds(None if ends is None else ends.cpu().numpy(), experts, rows)):
        for r in range(lo, hi):
            if r == 1:
                assert bool(got[r].isnan().all())
                continue
            exact, size = t.from_numpy(w[e] @ a[r]), t.from_numpy(np.abs(w[e]) @ np.abs(a[r]))
            check(got[r].cpu(), exact, size, (k / 64 + 64) * 2.0 ** -23, name)
    # rows further apart, and results too
    wide, out = t.zeros((rows, k + 5), dtype=x.dtype, device=gpu.dev), t.full((rows, n + 3), 5.0, dtype=x.dtype, device=gpu.dev)
    wide[:, :k] = x
    gpu.b.spinner_mx_linear(wide[:, :k], wc, ws, d, block, ends, out[:, :n])
    assert t.equal(out[:, :n].nan_to_num(nan=12345.0), got.nan_to_num(nan=12345.0)) and bool((out[:, n:] == 5).all())
    assert bool((gpu.b.spinner_mx_linear(x[:1].expand(rows, k), wc, ws, d, block, ends)[:1] == got[:1]).all())


def test_layers_of_few_rows_need_no_workspace(gpu):
    say("few rows, no workspace")
    t, b = gpu.torch, gpu.b
    d, w = t.ones(1024, device=gpu.dev), t.randn((48, 1024), device=gpu.dev)
    wc, ws = b.spinner_mx_quantize(w, d, 1024)
    for rows, status in ((4, b.SPINNER_OK), (5, b.SPINNER_ERR_WORKSPACE)):
        x, out = t.randn((rows, 1024), device=gpu.dev).bfloat16(), t.full((rows, 48), 5.0, device=gpu.dev).bfloat16()
        before = out.clone()
        rc = b.lib.spinner_mx_linear(x.data_ptr(), 1, rows, 1024, 1024, d.data_ptr(), 1024, wc.data_ptr(), ws.data_ptr(), 48, 1, None, out.data_ptr(), 48, None,
                                     b._stream_handle(None))
        assert rc == status
        assert t.equal(out, b.spinner_mx_linear(x, wc, ws, d, 1024) if rc == b.SPINNER_OK else before)
