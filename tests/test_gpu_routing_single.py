"""Renormalised rows of one choice: the weight is the scale and the gradient 0, whatever the score, as the quotient of a number and itself is 1."""
import numpy as np
import pytest

from oracle import experts_oracle as ex
from test_gpu_routing import gpu, held, numbers, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows,count", [(500, 60), (500, 999), (3000, 64), (3000, 250), (3000, 1000), (33000, 30), (33000, 64)])
def test_one_choice(gpu, rows, count, score, name):
    say("one choice", name, score, rows, count)
    rng = np.random.default_rng(rows + count)
    t = gpu.torch
    x = 3.0 * rng.standard_normal((rows, count))
    b, be = held(gpu, 0.1 * rng.standard_normal(count))
    for scale in (1.0, 2.5):
        for bias, bx in ((None, None), (b, be)):
            xt, xe = held(gpu, x, name)
            w, e = gpu.b.spinner_route(xt, 1, bias, None, score, scale=scale)
            assert bool((w == scale).all())
            d, _ = held(gpu, rng.standard_normal((rows, 1)))
            assert bool((gpu.b.spinner_route_grad(d, xt, e, score, scale=scale) == 0).all())
            # three choices, of which a row has one
            only = np.where(np.arange(count) == rng.integers(0, count, rows)[:, None], x, -np.inf)
            xt, xe = held(gpu, only, name)
            w, e = gpu.b.spinner_route(xt, 3, bias, None, score, scale=scale)
            some = slice(0, 50)
            assert np.array_equal(numbers(e)[some], ex.route(xe[some], 3, bx, None, score)[1])
            assert bool((w[:, 0] == scale).all()) and bool((w[:, 1:] == 0).all())
            d, _ = held(gpu, rng.standard_normal((rows, 3)))
            assert bool((gpu.b.spinner_route_grad(d, xt, e, score, scale=scale) == 0).all())
