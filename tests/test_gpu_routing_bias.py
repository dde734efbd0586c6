"""Routers whose biases are far from their scores: experts switched off or forced by a large finite number or by an infinity, against the 64-bit definitions.
Tolerances as in test_gpu_routing.py."""
import numpy as np
import pytest

from oracle import experts_oracle as ex
from test_gpu_routing import check_weights, gpu, held, numbers, say  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, experts, choices, groups, groups that stay: 64, 16 and four lanes a row
SIZES = [(40, 64, 8, 8, 3), (21, 512, 6, 64, 9), (2100, 256, 8, 8, 4), (2060, 60, 3, 12, 5), (16400, 32, 4, 4, 2)]


def choices(gpu, x, xe, bias, some, top, **o):
    b, be = held(gpu, bias)
    w, e = gpu.b.spinner_route(x, top, b, **o)
    want_w, want_e = ex.route(xe[some], top, be, None, **o)
    assert np.array_equal(numbers(e)[some], want_e), o
    check_weights(numbers(w)[some], want_w, xe, xe.shape[1])


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_biases_far_from_the_scores(gpu, case, score):
    rows, count, top, groups, top_groups = SIZES[case]
    say("far biases", SIZES[case], score)
    rng = np.random.default_rng(case)
    # few logits, so that scores and sums of them lie level or next to each other
    x, xe = held(gpu, rng.integers(-4, 5, (rows, count)) * 0.5 + rng.integers(0, 2, (rows, count)) * 2.0 ** -20)
    some = np.unique(np.concatenate((np.arange(12), rng.integers(0, rows, 40))))
    ordinary = 0.1 * rng.standard_normal(count)
    for far in (-1e9, -3e38, -1e4, 1e9, 3e38, np.inf, -np.inf):
        one, few, group = ordinary.copy(), ordinary.copy(), ordinary.copy()
        one[rng.integers(0, count)] = far
        few[rng.random(count) < 0.3] = far
        group[:count // groups] = far                        # a whole group
        for bias in (one, few, group):
            for o in ({}, dict(groups=groups, top_groups=top_groups, group_top=2), dict(groups=groups, top_groups=top_groups, group_top=1)):
                choices(gpu, x, xe, bias, some, top, score=score, **o)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_sums_of_two_keys_that_cancel_or_leave_32_bits(gpu, score):
    """Groups whose two largest keys are large and of either sign, and such whose sum is beyond fp32 but no infinity."""
    say("sums of large keys", score)
    rng = np.random.default_rng(3)
    count, groups, size = 64, 16, 4
    x, xe = held(gpu, 0.5 * rng.standard_normal((60, count)))
    some = np.arange(60)
    for large in (1e3, 1e6, 1e9):
        # one expert of each group far up, the second as far down, the others further: what is left is the scores'
        bias = np.tile([large, -large, -2 * large, -np.inf], groups) * rng.choice([1.0, 1.0 + 2.0 ** -20], groups).repeat(size)
        choices(gpu, x, xe, bias, some, 12, score=score, groups=groups, top_groups=4, group_top=2)
    # sums beyond fp32, up and down, in the order of their groups and against it
    for sign in (1.0, -1.0):
        bias = sign * (2.0e38 + 1e37 * rng.permutation(groups).repeat(size) % 12e37 + 1e36 * rng.random(count))
        choices(gpu, x, xe, bias, some, 16, score=score, groups=groups, top_groups=4, group_top=2)
        bias[:24] = 0.1 * rng.standard_normal(24)
        choices(gpu, x, xe, bias, some, 16, score=score, groups=groups, top_groups=4, group_top=2)


def test_one_far_bias_does_not_slow_the_others(gpu):
    """An expert switched off by a large number, or forced by one or by an infinity, costs no more than one of bias -inf: keys that 32 bits tell apart are not taken again."""
    say("far biases, time")
    t = gpu.torch
    g = t.Generator(device=gpu.dev).manual_seed(1)
    x = (1.5 * t.randn((16384, 256), generator=g, device=gpu.dev)).bfloat16()
    ordinary = 0.05 * t.randn(256, generator=g, device=gpu.dev)

    def time(bias, o):
        def call():
            gpu.b.spinner_route(x, 8, bias, None, "sigmoid", **o)
        best = 1e9
        for _ in range(5):
            a, b = t.cuda.Event(enable_timing=True), t.cuda.Event(enable_timing=True)
            call()
            a.record()
            for _ in range(20):
                call()
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) / 20)
        return best

    ratios = {}
    for o in ({}, dict(groups=8, top_groups=4, group_top=2)):
        times = {}
        for far in (-np.inf, -1e9, -1e6, 1e9, np.inf):
            bias = ordinary.clone()
            bias[100] = far
            times[far] = time(bias, o)
        say("ms", o, {k: round(v, 4) for k, v in times.items()})
        ratios.update({(len(o), far): times[far] / times[-np.inf] for far in times})
    # the slow forms take three times as long and more
    assert max(ratios.values()) < 1.5, ratios
