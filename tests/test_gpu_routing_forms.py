"""Routers of many rows and of every width: each form of the kernels (lanes a row, experts a lane), and rows whose keys lie level with each other, against the
64-bit definitions.  Tolerances as in test_gpu_routing.py."""
import numpy as np
import pytest

from oracle import experts_oracle as ex
from test_gpu_routing import check_grad, check_weights, gpu, held, numbers, say  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, experts, choices, groups, groups that stay: four lanes a row (8 and 16 experts each), 16 lanes (1, 4, 8, 16), 64 (1, 4, 8, 16, 32)
FORMS = [(2300, 7, 3, 1, 1), (2049, 32, 8, 1, 1), (2100, 61, 5, 1, 1), (2100, 64, 8, 4, 2), (2060, 48, 2, 3, 1), (2050, 40, 9, 1, 1), (2050, 16, 16, 1, 1), (2070, 13, 12, 1, 1), (2050, 100, 8, 4, 3),
         (2050, 128, 10, 8, 4), (2050, 256, 6, 16, 5), (2050, 250, 20, 10, 7), (33, 60, 4, 1, 1), (33, 64, 4, 64, 10), (20, 200, 7, 5, 2), (20, 400, 7, 50, 9), (20, 999, 9, 3, 2), (9, 1000, 30, 40, 25),
         (2050, 320, 4, 64, 6), (16390, 7, 3, 1, 1), (16384, 30, 4, 1, 1), (16385, 64, 4, 4, 2), (32770, 32, 8, 1, 1), (32768, 61, 5, 1, 1), (33000, 64, 8, 4, 3), (32800, 48, 6, 3, 2)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(FORMS)))
def test_each_form(gpu, name, case):
    rows, count, top, groups, top_groups = FORMS[case]
    say("route forms", name, FORMS[case])
    rng = np.random.default_rng(100 + case)
    t = gpu.torch
    x, xe = held(gpu, 2.0 * rng.standard_normal((rows, count)), name)
    b, be = held(gpu, 0.2 * rng.standard_normal(count))
    mask = rng.random(rows) < 0.9
    m = t.from_numpy(mask).to(gpu.dev)
    some = np.unique(np.concatenate((np.arange(min(rows, 40)), rng.integers(0, rows, 120), np.arange(max(0, rows - 30), rows))))
    for score, bias, group_top, renormalise in (("softmax", None, 1, False), ("sigmoid", be, 2, True), ("softmax", be, 1, True), ("sigmoid", None, 2, False)):
        o = dict(score=score, groups=groups, top_groups=top_groups, group_top=group_top, renormalise=renormalise)
        w, e = gpu.b.spinner_route(x, top, None if bias is None else b, m, **o)
        want_w, want_e = ex.route(xe[some], top, bias, mask[some], **o)
        assert np.array_equal(numbers(e)[some], want_e), o
        check_weights(numbers(w)[some], want_w, xe, count)
        d, de = held(gpu, rng.standard_normal((rows, top)))
        got = gpu.b.spinner_route_grad(d, x, e, score, renormalise)
        check_grad(numbers(got)[some], ex.route_grad(de[some], xe[some], want_e, score, renormalise), de[some], xe, count, 1.0, name)


@pytest.mark.parametrize("rows", [25, 2100, 33000])
@pytest.mark.parametrize("count,top", [(24, 8), (64, 8), (200, 12), (1000, 32)])
def test_keys_level_with_each_other(gpu, rows, count, top):
    """All equal, a few values only, and so near that fp32 does not tell them apart: more of them than a row's candidates; ties by index."""
    say("route level", rows, count, top)
    rng = np.random.default_rng(count)
    kinds = np.arange(rows) % 5
    x = np.zeros((rows, count))
    x[kinds == 1] = rng.integers(0, 3, (int((kinds == 1).sum()), count)) * 0.5
    x[kinds == 2] = 1.0 + rng.integers(0, 4, (int((kinds == 2).sum()), count)) * 2.0 ** -23
    x[kinds == 3] = np.where(rng.random((int((kinds == 3).sum()), count)) < 0.5, 0.0, -0.0)
    x[kinds == 4] = rng.integers(0, 2, (int((kinds == 4).sum()), count)) * 2.0 ** -149
    some = np.unique(np.concatenate((np.arange(25), rng.integers(0, rows, 40))))
    x, xe = held(gpu, x)
    biases = [None, np.zeros(count), (rng.integers(0, 2, count) * 2.0 ** -26).astype(np.float64)]
    for bias in biases:
        b, be = held(gpu, bias) if bias is not None else (None, None)
        for score in ("sigmoid", "softmax"):
            for groups in ({}, dict(groups=4, top_groups=3, group_top=2)):
                w, e = gpu.b.spinner_route(x, top, b, None, score, **groups)
                want_w, want_e = ex.route(xe[some], top, be, None, score, **groups)
                assert np.array_equal(numbers(e)[some], want_e), (score, groups)
                check_weights(numbers(w)[some], want_w, xe, count)


def test_scores_too_small_for_32_bits(gpu):
    """Logits of -90 to -700: their scores, and sums of two of them, decide all the same."""
    say("route small scores")
    rng = np.random.default_rng(5)
    x, xe = held(gpu, -90.0 - rng.integers(0, 600, (60, 64)))
    b, be = held(gpu, np.zeros(64))
    for score in ("sigmoid", "softmax"):
        for bias, bx in ((None, None), (b, be)):
            for groups in ({}, dict(groups=8, top_groups=3, group_top=2), dict(groups=8, top_groups=3, group_top=1)):
                w, e = gpu.b.spinner_route(x, 5, bias, None, score, **groups)
                want_w, want_e = ex.route(xe, 5, bx, None, score, **groups)
                assert np.array_equal(numbers(e), want_e), (score, groups)
                check_weights(numbers(w), want_w, xe, 64)


@pytest.mark.parametrize("rows", [400, 5000, 33000])
@pytest.mark.parametrize("far", [40.0, 66.0, 74.0, 87.3])
def test_scores_far_below_the_largest(gpu, rows, far):
    """One logit `far` above all others, which differ by a few places, and biases as small as their scores are: what fp32 rounds there decides nothing."""
    say("route far", rows, far)
    rng = np.random.default_rng(int(far) + rows)
    count, top = 64, 8
    x = -0.1 + rng.integers(0, 2000, (rows, count)) * 2.0 ** -27
    x[np.arange(rows), rng.integers(0, count, rows)] = far
    x, xe = held(gpu, x)
    some = np.unique(np.concatenate((np.arange(200), rng.integers(0, rows, 200))))
    small = np.exp(-far - 0.1)
    for bias in (np.zeros(count), rng.random(count) * small * 1e-5, -small * (1 + 1e-5 * rng.random(count))):
        b, be = held(gpu, bias)
        for groups in ({}, dict(groups=4, top_groups=2, group_top=2), dict(groups=4, top_groups=2, group_top=1)):
            w, e = gpu.b.spinner_route(x, top, b, None, "softmax", **groups)
            want_w, want_e = ex.route(xe[some], top, be, None, "softmax", **groups)
            assert np.array_equal(numbers(e)[some], want_e), groups
            check_weights(numbers(w)[some], want_w, xe, count)


def test_rows_beyond_32_bits(gpu):
    """Logits, rows at their places and codes whose offsets pass 2^31 bytes and numbers: the last rows as the first."""
    say("far rows")
    t, b = gpu.torch, gpu.b
    rows, count = 2200000, 1024
    x = t.empty((rows, count), dtype=t.bfloat16, device=gpu.dev)                    # 4.5 GB
    head = t.randn((5, count), device=gpu.dev).bfloat16()
    x[:5], x[-5:] = head, head
    w, e = b.spinner_route(x[-5:], 8)
    whole_w, whole_e = b.spinner_route(x, 8, mask=t.arange(rows, device=gpu.dev) >= rows - 5)
    assert t.equal(whole_w[-5:], w) and t.equal(whole_e[-5:], e) and bool((whole_e[:-5] == -1).all())
    del whole_w, whole_e
    places = t.arange(rows, dtype=t.int32, device=gpu.dev).flip(0).view(rows, 1).contiguous()
    y = b.spinner_dispatch(x, places)
    assert t.equal(y[:5].flip(0), head) and t.equal(y[-5:].flip(0), head)
    z = b.spinner_combine(y, places)
    assert t.equal(z[-5:], head) and t.equal(z[:5], head)
    del y, z
    codes, scales = b.spinner_int_quantize(x, None, 0, places)
    c, s = b.spinner_int_quantize(head)
    assert t.equal(codes[:5].flip(0), c) and t.equal(codes[-5:].flip(0), c) and t.equal(scales[:5].flip(0), s) and t.equal(scales[-5:].flip(0), s)
    assert t.equal(b.spinner_int_dequantize(codes, scales, t.bfloat16)[:5].flip(0), b.spinner_int_dequantize(c, s, t.bfloat16))
