"""Calls that are given a stream, while the current stream still works on memory that it has let go of."""
import sys

import numpy as np
import pytest

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
    return g


def say(*a):
    print("\n[gpu-case]", *a, file=sys.stderr, flush=True)


def product_calls(g):
    t, b = g.torch, g.b
    gen = t.Generator(device=g.dev)
    gen.manual_seed(3)
    rand = lambda *s: t.randn(s, generator=gen, device=g.dev)                                      # noqa: E731
    x, w, d = rand(300, 1024), rand(3, 96, 1024), t.ones(1024, device=g.dev)
    wc, ws = (v.view(3, 96, -1) for v in b.spinner_mx_quantize(w.view(-1, 1024), d, 512))
    ac, as_ = b.spinner_mx_quantize(x, d, 512)
    ends = t.tensor([100, 100, 290], device=g.dev)
    h, hw, dy = x.bfloat16(), w.bfloat16(), rand(300, 96).bfloat16()
    long_dy, long_x = rand(4100, 40).bfloat16(), rand(4100, 264).bfloat16()
    return {
        "mx_quantize": lambda **k: b.spinner_mx_quantize(x, d, 512, **k),
        "mx_dequantize": lambda **k: b.spinner_mx_dequantize(ac, as_, **k),
        "mx_matmul": lambda **k: b.spinner_mx_matmul(ac, as_, wc, ws, ends, **k),
        "mx_linear": lambda **k: b.spinner_mx_linear(h, wc, ws, d, 512, ends, **k),
        "grouped_matmul": lambda **k: b.spinner_grouped_matmul(h, hw, ends, **k),
        "grouped_matmul_dx": lambda **k: b.spinner_grouped_matmul_dx(dy, hw, ends, **k),
        "grouped_matmul_dw": lambda **k: b.spinner_grouped_matmul_dw(long_dy, long_x, **k),
    }


PRODUCTS = ["mx_quantize", "mx_dequantize", "mx_matmul", "mx_linear", "grouped_matmul", "grouped_matmul_dx", "grouped_matmul_dw"]


def check_call(g, call, monkeypatch):
    t = g.torch
    first = call()
    want = [r.clone() for r in (first if isinstance(first, tuple) else (first,))]
    t.cuda.synchronize()
    # blocks of the call's sizes that the current stream has let go of, and goes on writing to for a while
    made = []
    empty, empty_like = t.empty, t.empty_like

    def noted(make):
        def f(*a, **k):
            made.append(make(*a, **k))
            return made[-1]
        return f

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    late = [t.full((64 << 20,), 7.0, device=g.dev) for _ in range(2)]
    for k in range(8):
        late[k & 1].fill_(k)
    del first
    busy = [t.empty_like(r).fill_(3) for r in want]
    del busy, late
    with monkeypatch.context() as m:
        m.setattr(t, "empty", noted(empty))
        m.setattr(t, "empty_like", noted(empty_like))
        m.setattr(g.b, "_new_on", noted(g.b._new_on))
        got = call(stream=side)
    places = [(m.data_ptr(), m.numel()) for m in made]
    side.synchronize()
    for p, q in zip(got if isinstance(got, tuple) else (got,), want):
        assert t.equal(p, q)
    # what was made for the call lies in memory of its stream
    parts = [(s["address"], s["address"] + s["total_size"], s["stream"]) for s in t.cuda.memory_snapshot()]
    assert places
    for at, numel in places:
        if numel:
            assert [stream for lo, hi, stream in parts if lo <= at < hi] == [side.cuda_stream]


@pytest.mark.parametrize("name", PRODUCTS)
def test_products_on_a_stream_of_their_own(gpu, name, monkeypatch):
    say("stream of its own", name)
    check_call(gpu, product_calls(gpu)[name], monkeypatch)


def test_results_of_a_stream_outlive_what_the_current_one_reads_of_them(gpu):
    """A result that was made on another stream, let go of while the current one still reads it: not given away before."""
    say("results let go of early")
    t, b = gpu.torch, gpu.b
    x = t.randn((2048, 4096), device=gpu.dev).bfloat16()
    w = t.randn((4096, 4096), device=gpu.dev).bfloat16()
    side, wants, reads = t.cuda.Stream(), [], []
    for k in range(6):
        v = x * (k + 1)
        wants.append(b.spinner_grouped_matmul(v, w).double().sum(1))
        side.wait_stream(t.cuda.current_stream())
        y = b.spinner_grouped_matmul(v, w, stream=side)
        v.record_stream(side)
        t.cuda.current_stream().wait_stream(side)
        reads.append(y.double().sum(1))
        del y
        b.spinner_grouped_matmul(x, w, stream=side)          # may come to lie there, after the read
    t.cuda.synchronize()
    assert all(t.equal(p, q) for p, q in zip(reads, wants))
    assert np.isfinite(reads[0].cpu().numpy()).all()


def transform_calls(g):
    t, b = g.torch, g.b
    gen = t.Generator(device=g.dev)
    gen.manual_seed(4)
    n, wide = 1 << 12, 1 << 17
    x, xw = t.randn((300, n), generator=gen, device=g.dev), t.randn((9, wide), generator=gen, device=g.dev)
    d, dw = (t.randint(0, 2, (2, 3, s), generator=gen, device=g.dev).float() * 2 - 1 for s in (n, wide))
    signs, signs_w = b.spinner_pack_signs(d), b.spinner_pack_signs(dw)
    codes = b.spinner_sign_codes(x, *d[0])
    y, saved = b.spinner_layer_forward(x, *d[0], 0.5)
    gp = t.randn(n, generator=gen, device=g.dev)
    spectrum = b.spinner_struct_prepare("circulant", gp, n)
    A = t.randn((n, 60), generator=gen, device=g.dev)
    t.cuda.synchronize()
    return {
        "apply": lambda **k: b.spinner_apply(xw, *dw[0], 100, **k),
        "apply_signs": lambda **k: b.spinner_apply_signs(xw, signs_w, 100, **k),
        "apply_blocks": lambda **k: b.spinner_apply_blocks(x, d, 512, "cossin", 3.0, **k),
        "pack_signs": lambda **k: b.spinner_pack_signs(d, **k),
        "hash": lambda **k: b.spinner_hash(x, d, **k),
        "hash_signs": lambda **k: b.spinner_hash_signs(x, signs, 2, **k),
        "hash_ws": lambda **k: b.spinner_hash_ws(xw, dw, **k),
        "hash_signs_ws": lambda **k: b.spinner_hash_signs_ws(xw, signs_w, 2, **k),
        "sign_codes": lambda **k: b.spinner_sign_codes(xw, *dw[0], **k),
        "sign_codes_signs": lambda **k: b.spinner_sign_codes_signs(x, signs, **k),
        "angular_gram": lambda **k: b.spinner_angular_gram(codes, codes[:50], n, **k),
        "layer_forward": lambda **k: b.spinner_layer_forward(x, *d[0], 0.5, **k),
        "layer_backward": lambda **k: b.spinner_layer_backward(y, x, saved, *d[0], 0.5, **k),
        "sketch": lambda **k: b.spinner_sketch(A, None, *d[0], 128, **k),
        "sketch_gram": lambda **k: b.spinner_sketch_gram(A, **k),
        "struct_prepare": lambda **k: b.spinner_struct_prepare("circulant", gp, n, **k),
        "struct_apply": lambda **k: b.spinner_struct_apply(x, "circulant", spectrum, *d[0, :2], **k),
        "struct_apply_ws": lambda **k: b.spinner_struct_apply_ws(x, "circulant", spectrum, *d[0, :2], **k),
    }


TRANSFORMS = ["apply", "apply_signs", "apply_blocks", "pack_signs", "hash", "hash_signs", "hash_ws", "hash_signs_ws", "sign_codes", "sign_codes_signs", "angular_gram",
              "layer_forward", "layer_backward", "sketch", "sketch_gram", "struct_prepare", "struct_apply", "struct_apply_ws"]


@pytest.mark.parametrize("name", TRANSFORMS)
def test_transforms_on_a_stream_of_their_own(gpu, name, monkeypatch):
    say("stream of its own", name)
    check_call(gpu, transform_calls(gpu)[name], monkeypatch)


def test_whatever_has_a_handle_is_a_stream(gpu):
    """A stream object that has the handle alone, the default stream while another one is current, and the current one itself."""
    say("streams by their handle")
    t, b = gpu.torch, gpu.b
    x, w = t.randn((40, 512), device=gpu.dev).bfloat16(), t.randn((64, 512), device=gpu.dev).bfloat16()
    want = b.spinner_grouped_matmul(x, w)
    t.cuda.synchronize()
    side = t.cuda.Stream()
    owner = lambda r: [s["stream"] for s in t.cuda.memory_snapshot() if s["address"] <= r.data_ptr() < s["address"] + s["total_size"]]          # noqa: E731
    r = b.spinner_grouped_matmul(x, w, stream=type("Handle", (), {"cuda_stream": side.cuda_stream})())
    side.synchronize()
    assert t.equal(r, want) and owner(r) == [side.cuda_stream]
    with t.cuda.stream(side):
        r = b.spinner_grouped_matmul(x, w, stream=t.cuda.default_stream())
        assert t.cuda.current_stream() == side
        t.cuda.default_stream().synchronize()
        assert t.equal(r, want) and owner(r) == [0]
        r = b.spinner_grouped_matmul(x, w, stream=side)
        assert t.equal(r, want) and owner(r) == [side.cuda_stream]
    t.cuda.synchronize()
    with pytest.raises(t.cuda.OutOfMemoryError):                     # refused memory is an error, and leaves the current stream as it was
        b._new_on((1 << 50,), t.uint8, 0, side.cuda_stream, False)
    assert t.cuda.current_stream() == t.cuda.default_stream()
