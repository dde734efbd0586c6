"""Routing, the order of the experts and the rows' way there and back, against the 64-bit definitions (oracle/experts_oracle.py).

Tolerances.  A weight is a ratio of exponentials in fp32: an exponential of an argument a (itself rounded) is off by (|a| + 4) 2^-24 of itself, a sum
of n of them by (n / 16 + 12) 2^-24 more in the lanes' order, quotient and scale by three roundings.  Choices, places and ends are compared
exactly.  Gradients: the same of the factors, times the sum of magnitudes that they are made of, and one rounding to the type."""
import sys

import numpy as np
import pytest

from oracle import experts_oracle as ex

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


def held(g, x, name="f32"):
    t = g.torch.from_numpy(np.ascontiguousarray(x)).to(g.types[name]).to(g.dev)
    return t, numbers(t)


def numbers(t):
    return t.cpu().numpy() if not t.is_floating_point() else t.double().cpu().numpy()


def spread(x, bias=None):
    f = np.where(np.isfinite(x), x, 0.0)
    return np.abs(f).max(initial=0.0) * 2


def check_weights(got, want, logits, count):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    rel = (2 * spread(logits) + count / 16 + 24) * 2.0 ** -24
    keep = ~np.isnan(want)
    assert np.all(np.abs(got - want)[keep] <= (np.abs(want) * rel + 1e-37)[keep]), np.abs(got - want)[keep].max()


def check_grad(got, want, d, logits, count, scale, name):
    rel = (4 * spread(logits) + count / 16 + 60) * 2.0 ** -24
    size = scale * np.abs(np.where(np.isfinite(d), d, 0)).sum(1, keepdims=True)
    bound = np.abs(want) * 1.01 * HALF_STEP[name] + size * rel + TINY[name]
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)


PLAIN = dict()
FULL = dict(score="sigmoid", bias=True, groups=4, top_groups=2, group_top=2, scale=2.5)
ROUTERS = [
    (1, 1, 1, PLAIN), (1, 8, 2, dict(score="sigmoid")), (3, 5, 5, dict(renormalise=False)), (17, 16, 3, dict(bias=True)), (33, 17, 4, dict(score="sigmoid", bias=True)),
    (65, 64, 8, FULL), (40, 60, 6, dict(groups=12, top_groups=5, group_top=2)), (40, 60, 6, dict(groups=30, top_groups=7, bias=True, renormalise=False)),
    (129, 128, 8, dict(groups=8, top_groups=3, group_top=1)), (100, 256, 8, {**FULL, "groups": 8, "top_groups": 4}), (70, 250, 32, dict(bias=True)),
    (31, 257, 7, dict(score="sigmoid", bias=True)), (20, 512, 16, dict(groups=64, top_groups=9, group_top=2)), (9, 999, 11, dict(bias=True)),
    (5, 1024, 32, dict(score="sigmoid", renormalise=False, groups=2, top_groups=1, group_top=2, bias=True)), (300, 200, 1, PLAIN),
]


def options(rng, kwargs, count, rows):
    o = dict(kwargs)
    bias = 0.3 * rng.standard_normal(count) if o.pop("bias", False) else None
    return o, bias


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", range(len(ROUTERS)))
def test_routers_and_their_gradients(gpu, name, case):
    rows, count, top, kwargs = ROUTERS[case]
    say("route", name, rows, count, top, kwargs)
    rng = np.random.default_rng(case)
    o, bias = options(rng, kwargs, count, rows)
    x, xe = held(gpu, 2.0 * rng.standard_normal((rows, count)), name)
    b, be = held(gpu, bias) if bias is not None else (None, None)
    mask = rng.random(rows) < 0.8 if case % 2 else None
    m = None if mask is None else gpu.torch.from_numpy(mask).to(gpu.dev)
    w, e = gpu.b.spinner_route(x, top, b, m, **o)
    want_w, want_e = ex.route(xe, top, be, mask, **o)
    assert np.array_equal(numbers(e), want_e)
    check_weights(numbers(w), want_w, xe, count)
    places, ends = gpu.b.spinner_route_order(e, count)
    want_p, want_ends = ex.order(want_e, count)
    assert np.array_equal(numbers(places), want_p) and np.array_equal(numbers(ends), want_ends)
    d, de = held(gpu, rng.standard_normal((rows, top)))
    back = {k: o[k] for k in ("score", "renormalise", "scale") if k in o}
    got = gpu.b.spinner_route_grad(d, x, e, **back)
    check_grad(numbers(got), ex.route_grad(de, xe, want_e, **back), de, xe, count, back.get("scale", 1.0), name)


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("grouped", [False, True])
def test_values_that_are_no_ordinary_numbers(gpu, name, score, grouped):
    """Logits of -inf, +inf, NaN, of the type's lowest and largest value, all equal; biases of both infinities."""
    say("route values", name, score, grouped)
    rng = np.random.default_rng(7)
    low, inf, nan = float(gpu.torch.finfo(gpu.types[name]).min), np.inf, np.nan
    count, top = 24, 6
    x = rng.standard_normal((14, count))
    x[0] = -inf
    x[1, 3:] = -inf
    x[2, 5] = nan
    x[3, 5] = inf
    x[4] = low
    x[5, 2:] = low
    x[6] = 0.25
    x[7, ::2] = -inf
    x[8, :12] = -inf
    x[9] = -low
    x[10, 4] = -low
    x[11, :] = 60000.0
    x[12] = -200.0 - np.arange(count)
    x[13, 1:] = -inf
    x, xe = held(gpu, x, name)
    biases = [None, np.where(np.arange(count) % 5 == 0, -inf, 0.1 * rng.standard_normal(count)), np.where(np.arange(count) == 7, inf, 0.0),
              np.where(np.arange(count) == 9, nan, 0.0)]
    groups = dict(groups=4, top_groups=2) if grouped else {}
    for bias in biases:
        b, be = held(gpu, bias) if bias is not None else (None, None)
        for group_top in (1, 2) if grouped else (1,):
            for renormalise in (True, False):
                w, e = gpu.b.spinner_route(x, top, b, None, score, renormalise=renormalise, group_top=group_top, **groups)
                want_w, want_e = ex.route(xe, top, be, None, score, renormalise=renormalise, group_top=group_top, **groups)
                # (ties of scores that only 64 bits tell apart, or not even those, are the definition's by key and index)
                assert np.array_equal(numbers(e), want_e), (group_top, renormalise)
                finite = np.where(np.abs(xe) < 1e30, xe, 0.0)
                check_weights(numbers(w), want_w, finite, count)
                d, de = held(gpu, rng.standard_normal((14, top)))
                got = numbers(gpu.b.spinner_route_grad(d, x, e, score, renormalise))
                sane = [r for r in range(14) if r not in (2, 3)]
                want = ex.route_grad(de, xe, want_e, score, renormalise)
                check_grad(got[sane], want[sane], de[sane], finite[sane], count, 1.0, name)


def test_keys_that_32_bits_do_not_tell_apart(gpu):
    """Scores and biases whose sums differ by less than fp32 holds: taken in the order of 64 bits."""
    say("near keys")
    rng = np.random.default_rng(8)
    rows, count = 400, 64
    x = rng.standard_normal((rows, count)).astype(np.float32).astype(np.float64)
    s = ex.scores(x, "sigmoid")
    # one bias for all rows: rows alike but for a few last places
    x = np.repeat(x[:1], rows, 0) + 1e-7 * rng.standard_normal((rows, count))
    xt, xe = held(gpu, x)
    bias = (0.9 - s[0]).astype(np.float32)
    b, be = held(gpu, bias)
    for o in (dict(score="sigmoid"), dict(score="sigmoid", groups=8, top_groups=3, group_top=2)):
        w, e = gpu.b.spinner_route(xt, 8, b, **o)
        want_w, want_e = ex.route(xe, 8, be, None, **o)
        assert np.array_equal(numbers(e), want_e)
        assert (np.diff(np.sort(np.take_along_axis(ex.scores(xe, "sigmoid") + be, want_e, 1), 1)) < 2.0 ** -24).any()


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_logits_of_any_stride(gpu, name):
    say("route strides", name)
    rng = np.random.default_rng(9)
    t = gpu.torch
    wide, we = held(gpu, rng.standard_normal((21, 77)), name)
    for x, xe in ((wide[:, :50], we[:, :50]), (wide[::3, :64], we[::3, :64]), (wide[:1, :33].expand(9, 33), np.repeat(we[:1, :33], 9, 0))):
        w, e = gpu.b.spinner_route(x, 4, score="sigmoid")
        want_w, want_e = ex.route(xe, 4, score="sigmoid")
        assert np.array_equal(numbers(e), want_e)
        check_weights(numbers(w), want_w, xe, 64)
        d, de = held(gpu, rng.standard_normal(w.shape))
        out = t.full((x.shape[0], x.shape[1] + 5), 7.0, dtype=x.dtype, device=gpu.dev)
        got = gpu.b.spinner_route_grad(d, x, e, "sigmoid", dlogits=out[:, :x.shape[1]])
        check_grad(numbers(got), ex.route_grad(de, xe, want_e, "sigmoid"), de, xe, 64, 1.0, name)
        assert (out[:, x.shape[1]:] == 7).all()


def test_gradient_for_choices_of_any_kind(gpu):
    """The same expert twice in a row, none, and numbers that are no experts."""
    say("route grad choices")
    rng = np.random.default_rng(10)
    x, xe = held(gpu, rng.standard_normal((40, 30)))
    e = rng.integers(-3, 33, (40, 5)).astype(np.int32)
    e[3] = 4
    e[4] = -1
    et = gpu.torch.from_numpy(e).to(gpu.dev)
    d, de = held(gpu, rng.standard_normal((40, 5)))
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            got = numbers(gpu.b.spinner_route_grad(d, x, et, score, renormalise, 1.5))
            want = ex.route_grad(de, xe, e, score, renormalise, 1.5)
            check_grad(got, want, de, xe, 30, 1.5, "f32")


ORDERS = [(1, 1, 1), (0, 4, 3), (5, 3, 2), (64, 1, 64), (1000, 8, 16), (1024, 8, 1024), (1025, 8, 5), (3000, 3, 257), (40000, 2, 64), (70001, 1, 1000), (65536, 8, 256), (300000, 7, 9)]


@pytest.mark.parametrize("rows,top,count", ORDERS)
def test_order_of_the_experts(gpu, rows, top, count):
    say("order", rows, top, count)
    rng = np.random.default_rng(rows + count)
    t = gpu.torch
    for low, high in ((0, count), (-1, count + 1), (count // 2, count // 2 + 1)):
        e = rng.integers(low, high, (rows, top)).astype(np.int32)
        places, ends = gpu.b.spinner_route_order(t.from_numpy(e).to(gpu.dev), count)
        flat = np.where((e >= 0) & (e < count), e, count).reshape(-1)
        order = np.argsort(flat, kind="stable")
        want = np.empty(flat.size, dtype=np.int64)
        want[order] = np.arange(flat.size)
        assert np.array_equal(numbers(places).reshape(-1), want)
        assert np.array_equal(numbers(ends), np.cumsum(np.bincount(flat, minlength=count + 1))[:count])


WAYS = [(1, 1, 1), (1, 8, 2048), (3, 2, 7), (5, 4, 8), (9, 5, 9), (33, 3, 33), (40, 8, 130), (100, 6, 1001), (17, 32, 260), (65, 4, 2056), (12, 7, 4099), (4, 3, 70000)]


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,top,n", WAYS)
def test_there_and_back_with_gradients(gpu, name, rows, top, n):
    say("exchange", name, rows, top, n)
    rng = np.random.default_rng(rows + top + n)
    t = gpu.torch
    p = rng.permutation(rows * top).reshape(rows, top).astype(np.int32)
    places = t.from_numpy(p).to(gpu.dev)
    x, xe = held(gpu, rng.standard_normal((rows, n)), name)
    y, ye = held(gpu, rng.standard_normal((rows * top, n)), name)
    w, we = held(gpu, rng.standard_normal((rows, top)))
    assert np.array_equal(numbers(gpu.b.spinner_dispatch(x, places)), ex.dispatch(xe, p))
    for weights, wx in ((w, we), (None, None)):
        got, want = numbers(gpu.b.spinner_combine(y, places, weights)), ex.combine(ye, p, wx)
        size = ex.combine(np.abs(ye), p, None if wx is None else np.abs(wx))
        assert np.all(np.abs(got - want) <= np.abs(want) * 1.01 * HALF_STEP[name] + size * (top + 1) * 2.0 ** -24 + TINY[name])
    dy, dw = gpu.b.spinner_combine_grad(x, y, places, w)
    want_dy, want_dw = ex.combine_grad(xe, ye, p, we)
    assert np.all(np.abs(numbers(dy) - want_dy) <= np.abs(want_dy) * (1.01 * HALF_STEP[name] + 2.0 ** -24) + TINY[name])
    size = ex.combine_grad(np.abs(xe), np.abs(ye), p, we)[1]
    assert np.all(np.abs(numbers(dw) - want_dw) <= size * n * 2.0 ** -24 + TINY["f32"])


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_rows_further_apart_and_repeated(gpu, name):
    say("exchange strides", name)
    rng = np.random.default_rng(11)
    t = gpu.torch
    rows, top, n = 23, 3, 300
    p = rng.permutation(rows * top).reshape(rows, top).astype(np.int32)
    places = t.from_numpy(p).to(gpu.dev)
    wide, we = held(gpu, rng.standard_normal((rows * top, 511)), name)
    w, wx = held(gpu, rng.standard_normal((rows, top)))
    plain = {}
    for cut in (lambda a, r: a[:r, :n], lambda a, r: a[:1, :n].expand(r, n)):
        x, y = cut(wide, rows), cut(wide, rows * top)
        out = t.full((rows * top, 505), 5.0, dtype=x.dtype, device=gpu.dev)
        gpu.b.spinner_dispatch(x, places, out=out[:, :n])
        assert t.equal(out[:, :n], gpu.b.spinner_dispatch(x.contiguous(), places)) and (out[:, n:] == 5).all()
        back = t.full((rows, 303), 5.0, dtype=x.dtype, device=gpu.dev)
        gpu.b.spinner_combine(y, places, w, out=back[:, :n])
        assert t.equal(back[:, :n], gpu.b.spinner_combine(y.contiguous(), places, w)) and (back[:, n:] == 5).all()
        out.fill_(5.0)
        dy, dw = gpu.b.spinner_combine_grad(x, y, places, w, dy=out[:, :n])
        dy2, dw2 = gpu.b.spinner_combine_grad(x.contiguous(), y.contiguous(), places, w)
        assert t.equal(out[:, :n], dy2) and t.equal(dw, dw2) and (out[:, n:] == 5).all()


def test_places_outside_and_rows_that_are_not_to_be_read(gpu):
    """Places that are none are passed over, rows that none names stay as they were, and what has the weight 0 may hold anything."""
    say("exchange places")
    t = gpu.torch
    rng = np.random.default_rng(12)
    rows, top, n = 11, 2, 40
    p = rng.permutation(rows * top).reshape(rows, top).astype(np.int32)
    gone = [int(p[2, 1]), int(p[7, 0])]
    p[2, 1], p[7, 0] = -1, rows * top
    places = t.from_numpy(p).to(gpu.dev)
    x, xe = held(gpu, rng.standard_normal((rows, n)))
    y, ye = held(gpu, rng.standard_normal((rows * top, n)))
    w, we = held(gpu, rng.random((rows, top)) + 0.5)
    out = t.full((rows * top, n), 3.0, device=gpu.dev)
    gpu.b.spinner_dispatch(x, places, out=out)
    named = np.ones(rows * top, dtype=bool)
    named[gone] = False
    assert (out[gone] == 3).all() and np.array_equal(numbers(out)[[p[3, 0], p[2, 0]]], xe[[3, 2]])
    assert np.allclose(numbers(gpu.b.spinner_combine(y, places, w)), ex.combine(ye, p, we), atol=1e-6)
    dy = t.full((rows * top, n), 3.0, device=gpu.dev)
    dy, dw = gpu.b.spinner_combine_grad(x, y, places, w, dy=dy)
    assert (dy[gone] == 3).all() and dw[2, 1] == 0 and dw[7, 0] == 0
    assert np.allclose(numbers(dy)[named], ex.combine_grad(xe, ye, p, we)[0][named], atol=1e-6)
    w[0, 0] = 0
    y[int(p[0, 0])] = float("nan")
    assert t.equal(gpu.b.spinner_combine(y, places, w)[0], w[0, 1] * y[int(p[0, 1])])


def test_no_rows(gpu):
    t, b = gpu.torch, gpu.b
    w, e = b.spinner_route(t.zeros((0, 8), device=gpu.dev), 2)
    places, ends = b.spinner_route_order(e, 8)
    assert w.shape == e.shape == places.shape == (0, 2) and ends.tolist() == [0] * 8
    x = t.zeros((0, 16), device=gpu.dev)
    assert b.spinner_dispatch(x, places).shape == (0, 16) and b.spinner_combine(x, places, w).shape == (0, 16)
    assert b.spinner_route_grad(w, t.zeros((0, 8), device=gpu.dev), e).shape == (0, 8)
    assert [r.shape for r in b.spinner_combine_grad(x, x, places, w)] == [(0, 16), (0, 2)]
