"""Routers' weights and gradients with a bound for each number by its own row, and in every form in fp16.

Tolerances.  An exponential of l - top is off by (|l - top| + 4) 2^-24 of itself: the argument by half a place, the function by 2^-22.  A sum of them is off by the mean
of that over its terms, no more than ln(count) + 4 (the mean argument of count shares is below ln(count)), and by (count / 16 + 12) 2^-24 from its own order; the
sigmoid's denominator by four places; quotient and scale by two.  Scores below e^-87 are 0 in fp32.  A gradient is made of the shares' products with d and their
sum: each term's error as above, relative to the row's sum of |d|."""
import math

import numpy as np
import pytest

import test_gpu_routing_forms as forms
from oracle import experts_oracle as ex
from test_gpu_routing import HALF_STEP, TINY, gpu, held, numbers, say  # noqa: F401

pytestmark = pytest.mark.gpu


def arguments(x, experts, score, renormalise):
    """|argument| of the exponential of every choice, at most 90 (beyond, a score is 0)."""
    rows, count = x.shape
    l = np.take_along_axis(x, np.clip(experts, 0, count - 1), 1)
    l = np.where(experts >= 0, np.where(score == "sigmoid", np.minimum(l, 0.0), l), -np.inf)
    if renormalise:
        top = l.max(1, keepdims=True)
    else:
        top = np.zeros((rows, 1)) if score == "sigmoid" else x.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        a = np.abs(l - top)
    return np.where(np.isfinite(a), np.minimum(a, 90.0), 90.0 * (experts >= 0))


def check(g, x, xe, bias, mask, top, name, rng, **o):
    rows, count = xe.shape
    score, renormalise = o.get("score", "softmax"), o.get("renormalise", True)
    b, be = held(g, bias) if bias is not None else (None, None)
    w, e = g.b.spinner_route(x, top, b, mask, **o)
    want_w, want_e = ex.route(xe, top, be, None if mask is None else numbers(mask), **o)
    assert np.array_equal(numbers(e), want_e)
    a = arguments(xe, want_e, score, renormalise)
    keep = ~np.isnan(want_w)
    assert np.array_equal(np.isnan(numbers(w)), ~keep)
    rel = (a + 4 + math.log(count) + 4 + count / 16 + 12 + 4 + 2) * 2.0 ** -24
    off = np.abs(numbers(w) - want_w)
    assert np.all(off[keep] <= (np.abs(want_w) * rel + 1e-37)[keep]), np.max(off[keep] / (np.abs(want_w) * 2.0 ** -24 + 1e-37)[keep])
    d, de = held(g, rng.standard_normal((rows, top)))
    back = {k: o[k] for k in ("score", "renormalise", "scale") if k in o}
    got, want = numbers(g.b.spinner_route_grad(d, x, e, **back)), ex.route_grad(de, xe, want_e, **back)
    sane = keep.all(1)
    # (two factors of shares, or a share and 1 - p, of which the largest argument counts; products and the sum over the choices)
    far = a.max(1, initial=0.0)[:, None]
    rel = (2 * (far + 4 + math.log(count) + 4 + count / 16 + 12 + 4) + top + 4) * 2.0 ** -24
    size = o.get("scale", 1.0) * np.abs(de).sum(1, keepdims=True)
    bound = np.abs(want) * 1.01 * HALF_STEP[name] + size * rel + TINY[name]
    assert np.all((np.abs(got - want) <= bound)[sane]), np.max((np.abs(got - want) / bound)[sane])


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows", [1, 200, 1400])
def test_ordinary_rows_beside_others(gpu, rows, score, name):
    """Rows of unit size, of equal logits, of the type's largest and lowest values, with -inf among them, side by side."""
    say("rows by themselves", name, score, rows)
    rng = np.random.default_rng(rows)
    low, inf = float(gpu.torch.finfo(gpu.types[name]).min), np.inf
    count, top = 24, 6
    x = np.tile(rng.standard_normal((14, count)), (rows, 1)) if rows > 1 else rng.standard_normal((14, count))
    x += 0.5 * rng.standard_normal(x.shape)
    x[0::14] = -inf
    x[1::14, 3:] = -inf
    x[4::14] = low
    x[5::14, 2:] = low
    x[6::14] = 0.25
    x[7::14, ::2] = -inf
    x[8::14, :12] = -inf
    x[9::14] = -low
    x[10::14, 4] = -low
    x[11::14, :] = 60000.0
    x[12::14] = -200.0 - np.arange(count)
    x[13::14, 1:] = -inf
    some = np.arange(min(len(x), 56))
    xt, xe = held(gpu, x, name)
    for bias in (None, 0.1 * rng.standard_normal(count)):
        for renormalise in (True, False):
            for groups in ({}, dict(groups=4, top_groups=2, group_top=2)):
                check(gpu, xt[:some.size], xe[some], bias, None, top, name, rng, score=score, renormalise=renormalise, scale=1.5, **groups)
                # the same rows among many, which take another form: the same choices
                if rows > 1:
                    b = held(gpu, bias)[0] if bias is not None else None
                    w, e = gpu.b.spinner_route(xt, top, b, None, score, renormalise=renormalise, **groups)
                    w2, e2 = gpu.b.spinner_route(xt[:some.size], top, b, None, score, renormalise=renormalise, **groups)
                    assert gpu.torch.equal(e[:some.size], e2) and gpu.torch.allclose(w[:some.size], w2, rtol=2e-5, atol=1e-37)


@pytest.mark.parametrize("case", range(len(forms.FORMS)))
def test_each_form_in_fp16(gpu, case):
    forms.test_each_form(gpu, "f16", case)
