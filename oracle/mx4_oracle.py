"""Plain 64-bit definitions of the 4-bit format and of the grouped products (numpy only; test infrastructure).

Nothing here shares code with the library: the rotation is a dense Hadamard matrix, a rounding is a search among the eight
values a code can stand for, a product is a matrix product of each expert's rows.
"""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def hadamard(b: int) -> np.ndarray:
    """L2-normalised Hadamard matrix in Sylvester order, by its recursion."""
    h = np.ones((1, 1))
    while h.shape[0] < b:
        h = np.block([[h, h], [h, -h]])
    return h / np.sqrt(b)


def rotate(x: np.ndarray, diag, block: int) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    if not block:
        return x
    if diag is not None:
        x = x * np.asarray(diag, dtype=np.float64)
    return (x.reshape(-1, block) @ hadamard(block).T).reshape(x.shape)


def scale_bytes(top: np.ndarray) -> np.ndarray:
    """Scale byte of blocks whose largest magnitude is ``top``."""
    top = np.asarray(top, dtype=np.float64)
    _, e = np.frexp(np.where(np.isfinite(top) & (top > 0), top, 1.0))       # top = m 2^e, 1/2 <= m < 1
    byte = np.clip(e - 1 - 2 + 127, 0, 254)
    byte = np.where(top == 0, 0, byte)
    return np.where(np.isfinite(top), byte, 255).astype(np.uint8)


def round_to_codes(u: np.ndarray) -> np.ndarray:
    """Codes of numbers in units of their scale: the nearest value, ties to the one with the even code, held at the ends."""
    a = np.abs(u)
    far = np.abs(np.minimum(a, 6.0)[..., None] - VALUES)
    near = far.min(-1, keepdims=True)
    tie = far == near
    order = np.where(tie, np.where(np.arange(8) % 2 == 0, 0, 1), 2)         # even codes first among the nearest
    return (np.argmin(order, -1) + 8 * np.signbit(u)).astype(np.uint8)


def quantize(v: np.ndarray):
    """codes [rows][k] (one a number) and scale bytes [rows][k / 32]."""
    b = np.asarray(v, dtype=np.float64).reshape(*v.shape[:-1], -1, BLOCK)
    with np.errstate(invalid="ignore"):
        top = np.where(np.isnan(b).any(-1), np.inf, np.abs(b).max(-1))
    byte = scale_bytes(top)
    u = np.where((byte == 255)[..., None], 0.0, b) * np.exp2(127.0 - byte)[..., None]
    return round_to_codes(u).reshape(v.shape), byte


def pack(codes: np.ndarray) -> np.ndarray:
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed: np.ndarray) -> np.ndarray:
    return np.stack((packed & 15, packed >> 4), -1).reshape(*packed.shape[:-1], -1)


def values(packed: np.ndarray, byte: np.ndarray) -> np.ndarray:
    """What packed codes and their scale bytes stand for."""
    c = unpack(packed)
    v = np.where(c & 8, -1.0, 1.0) * VALUES[c & 7]
    scale = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127.0))
    return v * np.repeat(scale, BLOCK, -1)


def bounds(ends, experts: int, rows: int):
    """[(lo, hi)] of the experts' rows, the ends held between 0 and ``rows`` and to rise."""
    if ends is None:
        return [(0, rows)] * experts
    found, before = [], 0
    for e in range(experts):
        hi = max(before, min(max(int(ends[e]), 0), rows))
        found.append((before, hi))
        before = hi
    return found


def products(x: np.ndarray, w: np.ndarray, ends=None) -> np.ndarray:
    """x w^T of each expert's rows, rows of no expert 0."""
    y = np.zeros((x.shape[0], w.shape[1]))
    for e, (lo, hi) in enumerate(bounds(ends, w.shape[0], x.shape[0])):
        y[lo:hi] = x[lo:hi] @ w[e].T
    return y


def products_dx(dy: np.ndarray, w: np.ndarray, ends=None) -> np.ndarray:
    return products(dy, np.swapaxes(w, 1, 2), ends)


def products_dw(dy: np.ndarray, x: np.ndarray, experts: int, ends=None) -> np.ndarray:
    return np.stack([dy[lo:hi].T @ x[lo:hi] for lo, hi in bounds(ends, experts, x.shape[0])])
