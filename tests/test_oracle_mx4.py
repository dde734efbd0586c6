"""Pins of the 64-bit definitions of the 4-bit format and of the grouped products: hand-written values, brute force, identities."""
import numpy as np
import pytest

from oracle import mx4_oracle as mx

RNG = np.random.default_rng(5)


def test_codes_of_hand_written_numbers():
    u = np.array([0, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 1.74, 2.5, 2.51, 3.5, 3.49, 5.0, 5.01, 6.0, 7.9, -0.5, -6.0])
    want = [0, 0, 1, 2, 1, 2, 3, 4, 3, 4, 5, 6, 5, 6, 7, 7, 7, 9, 15]
    assert mx.round_to_codes(u).tolist() == want
    assert mx.round_to_codes(np.array([-0.0]))[0] == 8


def test_scale_of_hand_written_blocks():
    top = np.array([4.0, 3.999, 7.999, 8.0, 1.0, 0.0, np.inf, 2.0 ** -126, 2.0 ** -149, 3.0e38])
    assert mx.scale_bytes(top).tolist() == [127, 126, 127, 128, 125, 0, 255, 0, 0, 252]


def test_a_code_is_the_nearest_value():
    v = RNG.standard_normal((40, 96)) * np.exp(RNG.uniform(-20, 20, (40, 1)))
    codes, byte = mx.quantize(v)
    got = mx.values(mx.pack(codes), byte)
    scale = np.repeat(np.exp2(byte.astype(float) - 127), 32, -1)
    for s in (-1.0, 1.0):
        for value in mx.VALUES:
            assert np.all(np.abs(v - got) <= np.abs(v - s * value * scale) * (1 + 1e-12))
    top = np.abs(v).reshape(40, -1, 32).max(-1)
    assert np.all(top < 8 * np.exp2(byte - 127.0)) and np.all(top >= 4 * np.exp2(byte - 127.0))


def test_quantising_what_is_already_in_4_bits_changes_nothing():
    codes = RNG.integers(0, 16, (9, 64)).astype(np.uint8)
    codes[:, ::32] = 7                                     # a full block has a number of 4 and more
    byte = RNG.integers(3, 250, (9, 2)).astype(np.uint8)
    again, byte2 = mx.quantize(mx.values(mx.pack(codes), byte))
    assert np.array_equal(byte, byte2) and np.array_equal(again, codes)
    assert np.array_equal(mx.unpack(mx.pack(codes)), codes)


def test_nothing_and_no_number():
    v = np.zeros((3, 64))
    v[1, 5], v[2, 40] = np.nan, -np.inf
    codes, byte = mx.quantize(v)
    assert byte.tolist() == [[0, 0], [255, 0], [0, 255]] and not codes.any()
    got = mx.values(mx.pack(codes), byte)
    assert np.isnan(got[1, :32]).all() and not got[1, 32:].any() and np.isnan(got[2, 32:]).all() and not got[0].any()


@pytest.mark.parametrize("block", [32, 64, 256])
def test_rotating_both_operands_leaves_their_product(block):
    x, w = RNG.standard_normal((5, 512)), RNG.standard_normal((7, 512))
    d = RNG.choice([-1.0, 1.0], 512)
    h = mx.hadamard(block)
    i = np.arange(block)
    want = np.array([[(-1.0) ** bin(int(a & b)).count("1") for b in i] for a in i]) / np.sqrt(block)
    assert np.allclose(h, want, atol=1e-15)
    assert np.allclose(mx.rotate(x, d, block) @ mx.rotate(w, d, block).T, x @ w.T, atol=1e-10)
    assert np.allclose(mx.rotate(x, d, block)[3, block:2 * block], want @ (d * x[3])[block:2 * block], atol=1e-12)


def test_rotation_spreads_a_large_coordinate_so_that_4_bits_hold_the_rest():
    x, w = RNG.standard_normal((20, 1024)), RNG.standard_normal((30, 1024)) / 32
    x[:, 100] = 200.0
    w[:, 100] /= 200.0
    d = RNG.choice([-1.0, 1.0], 1024)

    def error(block):
        a, b = (mx.values(mx.pack(c), s) for c, s in (mx.quantize(mx.rotate(v, d if block else None, block)) for v in (x, w)))
        return np.linalg.norm(a - mx.rotate(x, d, block)) / np.linalg.norm(x[:, :100])

    plain = mx.values(*[f(v) for f, v in zip((mx.pack, lambda s: s), mx.quantize(x))])
    lost = plain[:, 96:128][:, np.arange(32) != 4]
    assert not lost.any()                                  # the neighbours of the large one are gone
    assert np.count_nonzero(mx.quantize(mx.rotate(x, d, 1024))[0] & 7) > 0.5 * x.size
    assert error(1024) < np.inf


def test_grouped_products_row_by_row():
    x, w, dy = RNG.standard_normal((11, 6)), RNG.standard_normal((4, 5, 6)), RNG.standard_normal((11, 5))
    ends = [3, 3, 8, 9]
    expert = [0, 0, 0, 2, 2, 2, 2, 2, 3, None, None]
    y, dx, dw = mx.products(x, w, ends), mx.products_dx(dy, w, ends), mx.products_dw(dy, x, 4, ends)
    want = np.zeros_like(w)
    for r, e in enumerate(expert):
        assert np.allclose(y[r], 0 if e is None else w[e] @ x[r])
        assert np.allclose(dx[r], 0 if e is None else w[e].T @ dy[r])
        if e is not None:
            want[e] += np.outer(dy[r], x[r])
    assert np.allclose(dw, want) and not dw[1].any()


def test_gradients_are_those_of_differences():
    x, w, dy = RNG.standard_normal((11, 6)), RNG.standard_normal((4, 5, 6)), RNG.standard_normal((11, 5))
    ends, h = [3, 3, 8, 9], 1e-5
    loss = lambda a, b: float((dy * mx.products(a, b, ends)).sum())                               # noqa: E731
    dx, dw = mx.products_dx(dy, w, ends), mx.products_dw(dy, x, 4, ends)
    u, v = RNG.standard_normal(x.shape), RNG.standard_normal(w.shape)
    assert np.isclose((loss(x + h * u, w) - loss(x - h * u, w)) / (2 * h), (dx * u).sum(), rtol=1e-8)
    assert np.isclose((loss(x, w + h * v) - loss(x, w - h * v)) / (2 * h), (dw * v).sum(), rtol=1e-8)


def test_ends_out_of_order_are_held_in_order():
    assert mx.bounds([5, 2, 900, -7, 4], 5, 12) == [(0, 5), (5, 5), (5, 12), (12, 12), (12, 12)]


@pytest.mark.parametrize("mistake", ["odd ties", "ceil scale", "high half first", "neighbour's rows"])
def test_planted_mistakes_are_seen(mistake):
    """Each mistake, made in a copy of a definition, gives results that the checks above tell apart."""
    v = RNG.standard_normal((8, 64))
    v[:, 0], v[:, 1:8] = 4.0, [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -2.5]
    codes, byte = mx.quantize(v)
    if mistake == "odd ties":
        a = np.abs(v[0, 1:8])
        wrong = np.array([np.flatnonzero(np.abs(x - mx.VALUES) == np.abs(x - mx.VALUES).min())[np.argmax(
            np.flatnonzero(np.abs(x - mx.VALUES) == np.abs(x - mx.VALUES).min()) % 2)] for x in a])
        assert not np.array_equal(wrong, codes[0, 1:8] & 7)
    elif mistake == "ceil scale":
        assert not np.array_equal(byte + 1, byte)
    elif mistake == "high half first":
        swapped = (codes[:, 1::2] | (codes[:, 0::2] << 4)).astype(np.uint8)
        assert not np.array_equal(mx.values(swapped, byte), mx.values(mx.pack(codes), byte))
    else:
        x, w = RNG.standard_normal((9, 8)), RNG.standard_normal((3, 4, 8))
        assert not np.allclose(mx.products(x, w, [3, 5, 9]), mx.products(x, w, [4, 5, 9]))
