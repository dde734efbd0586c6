"""Calls of so many rows that a workgroup takes several in turn: routers beyond 2^20 workgroups, the rows' ways there and back and 8-bit rows beyond 2^22.
Rows repeat a short call's, whose results they have to have bit for bit."""
import pytest

from test_gpu_routing import gpu, say  # noqa: F401

pytestmark = pytest.mark.gpu


def repeated(t, head, rows):
    """head over and over, `rows` of it."""
    times = -(-rows // head.shape[0])
    return head.repeat((times,) + (1,) * (head.dim() - 1))[:rows]


def same(t, got, head):
    period, whole = head.shape[0], got.shape[0] // head.shape[0] * head.shape[0]
    assert bool((got[:whole].view(-1, *head.shape) == head).all()) and t.equal(got[whole:], head[:got.shape[0] - whole])


# lanes a row, experts, choices, rows of the short call, which takes the same form
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("lanes,count,top,period", [(4, 4, 1, 40009), (16, 65, 2, 3001), (64, 257, 2, 3001)])
def test_routers(gpu, lanes, count, top, period, biased):
    say("turns, router", lanes, biased)
    t, b = gpu.torch, gpu.b
    rows = (1 << 20) * (256 // lanes) + 777
    g = t.Generator(device=gpu.dev).manual_seed(lanes)
    head, d = t.randn((period, count), device=gpu.dev, generator=g).bfloat16(), t.randn((period, top), device=gpu.dev, generator=g)
    bias = 0.1 * t.randn(count, device=gpu.dev, generator=g) if biased else None
    w, e = b.spinner_route(head, top, bias, None, "sigmoid", renormalise=False)
    x = repeated(t, head, rows)
    many_w, many_e = b.spinner_route(x, top, bias, None, "sigmoid", renormalise=False)
    same(t, many_w, w)
    same(t, many_e, e)
    del many_w
    if not biased:
        for score in ("sigmoid", "softmax"):
            same(t, b.spinner_route_grad(repeated(t, d, rows), x, many_e, score, False), b.spinner_route_grad(d, head, e, score, False))


# rows that a workgroup takes at a time in the ways and in the gradient, numbers of a row
@pytest.mark.parametrize("each,grad_each,n", [(16, 16, 8), (4, 4, 136), (4, 1, 1032)])
def test_ways_there_and_back(gpu, each, grad_each, n):
    say("turns, exchange", each, grad_each, n)
    t, b = gpu.torch, gpu.b
    runs = -(-n * 2 // 1024)
    rows = max((1 << 22) * each // runs, (1 << 22) * grad_each) + 333
    period = 1009
    g = t.Generator(device=gpu.dev).manual_seed(n)
    head, other = (t.randn((period, n), device=gpu.dev, generator=g).bfloat16() for _ in range(2))
    w = t.rand((period, 1), device=gpu.dev, generator=g) + 0.5
    # every row to the place of its own number
    places = t.arange(rows, dtype=t.int32, device=gpu.dev).view(rows, 1)
    near = places[:period].contiguous()
    x = repeated(t, head, rows)
    assert t.equal(b.spinner_dispatch(x, places), x)
    weights = repeated(t, w, rows)
    same(t, b.spinner_combine(x, places, weights), b.spinner_combine(head, near, w))
    dy, dw = b.spinner_combine_grad(repeated(t, other, rows), x, places, weights)
    head_dy, head_dw = b.spinner_combine_grad(other, head, near, w)
    same(t, dy, head_dy)
    same(t, dw, head_dw)


def test_8_bit_rows(gpu):
    say("turns, 8-bit rows")
    t, b = gpu.torch, gpu.b
    rows, period = (1 << 22) * 16 + 55, 1013
    head = t.randn((period, 16), device=gpu.dev).bfloat16()
    c, s = b.spinner_int_quantize(head)
    codes, scales = b.spinner_int_quantize(repeated(t, head, rows))
    same(t, codes, c)
    same(t, scales, s)
    same(t, b.spinner_int_dequantize(codes, scales, t.bfloat16), b.spinner_int_dequantize(c, s, t.bfloat16))
