"""Pins of the 64-bit definitions of routing and of 8-bit rows: worked examples, differences, other formulas."""
import numpy as np
import pytest

from oracle import experts_oracle as ex


def test_a_worked_router():
    x = np.log(np.array([[1.0, 2.0, 4.0, 1.0]]))
    w, e = ex.route(x, 2, renormalise=False)
    assert e.tolist() == [[2, 1]] and np.allclose(w, [[0.5, 0.25]])
    w, e = ex.route(x, 2)
    assert np.allclose(w, [[2 / 3, 1 / 3]])
    # the bias takes part in the choice only; ties go to the lower index
    w, e = ex.route(x, 2, bias=np.array([0.4, 0, 0, 0.4]), renormalise=False, scale=2.0)
    assert e.tolist() == [[0, 3]] and np.allclose(w, [[0.25, 0.25]])
    w, e = ex.route(np.zeros((1, 3)), 2, score="sigmoid")
    assert e.tolist() == [[0, 1]] and np.allclose(w, 0.5)


def test_groups_of_a_worked_router():
    x = np.array([[3.0, 0, 2, 2, 1, 1]])
    kept = {(1, 1): [0, 1], (1, 2): [2, 3]}
    for (top_groups, group_top), want in kept.items():
        _, e = ex.route(x, 2, score="sigmoid", groups=3, top_groups=top_groups, group_top=group_top)
        assert e.tolist() == [want]
    _, e = ex.route(np.array([[-np.inf, 5.0, 1, 1]]), 3, groups=2, top_groups=2, group_top=2)
    assert e.tolist() == [[1, 2, 3]]


def test_rows_with_nothing_to_choose():
    x = np.array([[0.0, 1, 2], [-np.inf] * 3, [1, -np.inf, 0], [1, np.nan, 0], [0, 1, 2]])
    w, e = ex.route(x, 3, mask=[1, 1, 1, 1, 0])
    assert e.tolist() == [[2, 1, 0], [-1] * 3, [0, 2, -1], [-1] * 3, [-1] * 3]
    assert (w[1] == 0).all() and w[2, 2] == 0 and np.isnan(w[3]).all() and (w[4] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_gradient_of_the_weights_by_differences(score, renormalise):
    rng = np.random.default_rng(3)
    x, d, h = rng.standard_normal((4, 7)), rng.standard_normal((4, 3)), 1e-6
    w, e = ex.route(x, 3, score=score, renormalise=renormalise, scale=1.7)
    e[1, 2] = -1
    d0 = np.where(e >= 0, d, 0.0)

    def total(x):
        s = ex.scores(x, score)
        out = 0.0
        for r in range(4):
            mine = [j for j in range(3) if e[r, j] >= 0]
            chosen = np.array([s[r, e[r, j]] for j in mine])
            out += 1.7 * (chosen / (chosen.sum() if renormalise else 1.0) * d0[r, mine]).sum()
        return out

    want = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        step = np.zeros_like(x)
        step[i] = h
        want[i] = (total(x + step) - total(x - step)) / (2 * h)
    # differences of h = 1e-6: h^2 of the third derivative and 2^-53 / h of the sums
    assert np.abs(ex.route_grad(d, x, e, score, renormalise, 1.7) - want).max() < 1e-8


def test_places_are_a_stable_order():
    e = np.array([[2, 0], [-1, 2], [0, 9], [2, 1]])
    places, ends = ex.order(e, 3)
    assert places.tolist() == [[3, 0], [6, 4], [1, 7], [5, 2]] and ends.tolist() == [2, 3, 6]


def test_there_and_back():
    rng = np.random.default_rng(4)
    x, w = rng.standard_normal((5, 3)), rng.random((5, 2))
    places = rng.permutation(10).reshape(5, 2)
    y = ex.dispatch(x, places)
    assert np.allclose(ex.combine(y, places, w), x * w.sum(1, keepdims=True)) and np.allclose(ex.combine(y, places), 2 * x)
    dout, y = rng.standard_normal((5, 3)), rng.standard_normal((10, 3))
    dy, dw = ex.combine_grad(dout, y, places, w)
    # linear in y and in w: the gradient's product with either is the sum's with dout
    assert np.isclose((dy * y).sum(), (ex.combine(y, places, w) * dout).sum()) and np.isclose((dw * w).sum(), (dy * y).sum())


def test_rows_of_whole_numbers():
    x = np.array([[127.0, -63.5, 0.5, 1.5, -2.5, 0.49], [0, 0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0, 0]])
    codes, scale = ex.int_quantize(x)
    assert codes[0].tolist() == [127, -64, 0, 2, -2, 0] and scale[0] == 1 and scale[1] == np.float32(2.0 ** -126) and np.isnan(scale[2])
    assert not codes[1:].any()
    # off by at most half a step, and by a rotation that leaves products as they are
    rng = np.random.default_rng(5)
    v = rng.standard_normal((6, 64))
    codes, scale = ex.int_quantize(v, np.sign(rng.standard_normal(64)), 32)
    assert np.abs(codes).max() == 127
    codes, scale = ex.int_quantize(v)
    assert np.all(np.abs(codes * scale[:, None].astype(float) - v) <= 0.5 * scale[:, None] * (1 + 1e-12))
    out = ex.int_products(codes, scale, codes[None, :3], scale[None, :3])
    assert np.allclose(out, (codes * scale[:, None].astype(float)) @ (codes[:3] * scale[:3, None].astype(float)).T)
