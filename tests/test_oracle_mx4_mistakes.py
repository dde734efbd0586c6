"""That the pins of the 4-bit definitions fail when a definition is wrong: each mistake is made in the oracle, and the pins of test_oracle_mx4.py that should see it are run.
And what the rotation is for, in numbers."""
import numpy as np
import pytest

import test_oracle_mx4 as pins
from oracle import mx4_oracle as mx

RIGHT = {name: getattr(mx, name) for name in ("round_to_codes", "scale_bytes", "pack", "unpack", "values", "hadamard", "bounds", "quantize")}


def odd_ties(u):
    a = np.minimum(np.abs(u), 6.0)[..., None]
    order = np.where(np.abs(a - mx.VALUES) == np.abs(a - mx.VALUES).min(-1, keepdims=True), np.where(np.arange(8) % 2, 0, 1), 2)
    return (np.argmin(order, -1) + 8 * np.signbit(u)).astype(np.uint8)


def towards_zero(u):
    return (np.searchsorted(mx.VALUES, np.minimum(np.abs(u), 6.0), side="right") - 1 + 8 * np.signbit(u)).astype(np.uint8)


def no_sign_of_zero(u):
    code = RIGHT["round_to_codes"](u)
    return np.where(code == 8, 0, code).astype(np.uint8)


def next_power(top):
    return np.where(np.isfinite(top) & (top > 0), RIGHT["scale_bytes"](top).astype(int) + 1, RIGHT["scale_bytes"](top)).astype(np.uint8)


def rounded_power(top):
    byte = RIGHT["scale_bytes"](top).astype(int)
    mantissa = np.frexp(np.where(np.isfinite(top) & (top > 0), top, 1.0))[0]
    return np.where(np.isfinite(top) & (top > 0) & (mantissa > 0.75), np.minimum(byte + 1, 254), byte).astype(np.uint8)


def zeros_of_scale_one(top):
    return np.where(np.asarray(top) == 0, 127, RIGHT["scale_bytes"](top)).astype(np.uint8)


def no_byte_for_nan(top):
    return np.minimum(RIGHT["scale_bytes"](top), 254).astype(np.uint8)


def high_half_first(codes):
    return (codes[..., 1::2] | (codes[..., 0::2] << 4)).astype(np.uint8)


def no_nan(packed, byte):
    return RIGHT["values"](packed, np.where(byte == 255, 254, byte))


def not_normalised(b):
    return RIGHT["hadamard"](b) * np.sqrt(b)


def by_sequency(b):
    h = RIGHT["hadamard"](b)
    return h[np.argsort((np.diff(np.sign(h), axis=1) != 0).sum(1), kind="stable")]


def first_row_left_out(ends, experts, rows):
    return [(min(lo + 1, hi), hi) for lo, hi in RIGHT["bounds"](ends, experts, rows)]


def rows_of_none_to_the_last(ends, experts, rows):
    found = RIGHT["bounds"](ends, experts, rows)
    return found[:-1] + [(found[-1][0], rows)]


def ends_as_they_come(ends, experts, rows):
    return [(0 if e == 0 else int(ends[e - 1]), int(ends[e])) for e in range(experts)] if ends is not None else [(0, rows)] * experts


MISTAKES = {
    odd_ties: ("round_to_codes", pins.test_codes_of_hand_written_numbers),
    towards_zero: ("round_to_codes", pins.test_codes_of_hand_written_numbers, pins.test_a_code_is_the_nearest_value),
    no_sign_of_zero: ("round_to_codes", pins.test_codes_of_hand_written_numbers),
    next_power: ("scale_bytes", pins.test_scale_of_hand_written_blocks, pins.test_a_code_is_the_nearest_value, pins.test_quantising_what_is_already_in_4_bits_changes_nothing),
    rounded_power: ("scale_bytes", pins.test_scale_of_hand_written_blocks, pins.test_a_code_is_the_nearest_value),
    zeros_of_scale_one: ("scale_bytes", pins.test_scale_of_hand_written_blocks, pins.test_nothing_and_no_number),
    no_byte_for_nan: ("scale_bytes", pins.test_scale_of_hand_written_blocks, pins.test_nothing_and_no_number),
    high_half_first: ("pack", pins.test_a_code_is_the_nearest_value, pins.test_quantising_what_is_already_in_4_bits_changes_nothing),
    no_nan: ("values", pins.test_nothing_and_no_number),
    not_normalised: ("hadamard", lambda: pins.test_rotating_both_operands_leaves_their_product(64)),
    by_sequency: ("hadamard", lambda: pins.test_rotating_both_operands_leaves_their_product(64)),
    first_row_left_out: ("bounds", pins.test_grouped_products_row_by_row, pins.test_ends_out_of_order_are_held_in_order),
    rows_of_none_to_the_last: ("bounds", pins.test_grouped_products_row_by_row),
    ends_as_they_come: ("bounds", pins.test_ends_out_of_order_are_held_in_order),
}


@pytest.mark.parametrize("mistake", list(MISTAKES), ids=lambda f: f.__name__)
def test_a_mistake_in_a_definition_fails_its_pins(mistake, monkeypatch):
    name, *checks = MISTAKES[mistake]
    for check in checks:
        check()
    monkeypatch.setattr(mx, name, mistake)
    for check in checks:
        with pytest.raises(AssertionError):
            check()


def test_gradients_of_other_rows_are_seen_by_differences(monkeypatch):
    """A gradient whose groups are not those of the product."""
    monkeypatch.setattr(mx, "products_dx", lambda dy, w, ends: mx.products(dy, np.swapaxes(w, 1, 2), [e + 1 for e in ends]))
    with pytest.raises(AssertionError):
        pins.test_gradients_are_those_of_differences()


@pytest.mark.parametrize("large", [40.0, 60.0])
def test_the_rotation_lowers_the_error_of_what_is_not_large(large):
    """One coordinate of 1024 is large.  Without the rotation its block has the scale 2^(5 - 2) = 8: the 31 others, of standard deviation 1, become 0 up to a magnitude of 2, where
    three quarters of their energy lies, and 4 above it: a relative error of sqrt(0.74) = 0.86 and more.  With it every coordinate has the deviation s = sqrt(1 + large^2 / 1024), 2.1 for
    60, and an error of at most half the widest step, 2^e where the block's largest magnitude is 4 2^e to 8 2^e: under a quarter of that one, and under a quarter of s in the mean, as
    most numbers lie where the steps are a quarter as wide."""
    rng = np.random.default_rng(11)
    x = rng.standard_normal((50, 1024))
    x[:, 100] = large
    d = rng.choice([-1.0, 1.0], 1024)
    others = np.arange(1024) != 100
    beside = others & (np.arange(1024) // 32 == 100 // 32)
    h = mx.hadamard(1024)

    def held(v):
        codes, byte = mx.quantize(v)
        return mx.values(mx.pack(codes), byte)

    direct = held(x)
    back = (held(mx.rotate(x, d, 1024)) @ h) * d                     # H is its own inverse
    relative = lambda got, which: np.linalg.norm((got - x)[:, which]) / np.linalg.norm(x[:, which])          # noqa: E731
    spread = np.sqrt(1 + large ** 2 / 1024)
    assert relative(direct, beside) > 0.85
    assert relative(back, beside) < 0.25 * spread and relative(back, others) < 0.25 * spread
    # a product with weights that have use for the small ones
    w = rng.standard_normal((30, 1024))
    w[:, 100] /= large
    error = lambda a, b: np.linalg.norm(a @ b.T - x @ w.T) / np.linalg.norm(x @ w.T)                         # noqa: E731
    assert error(held(mx.rotate(x, d, 1024)), held(mx.rotate(w, d, 1024))) < 0.25 * np.hypot(spread, 1)
