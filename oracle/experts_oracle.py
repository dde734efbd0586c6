"""Plain 64-bit definitions of routing, of the rows' way to the experts and back, and of 8-bit rows (numpy only; test infrastructure).

Nothing here shares code with the library: rows are routed one by one by sorting, places are counted, sums are loops over the choices.
"""
from __future__ import annotations

import numpy as np

from .mx4_oracle import rotate

NONE = -1


def scores(logits: np.ndarray, score: str) -> np.ndarray:
    x = np.asarray(logits, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            return np.where(x > 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))
        top = x.max(-1, keepdims=True)
        e = np.where(x > -np.inf, np.exp(x - np.where(top > -np.inf, top, 0.0)), 0.0)
        total = e.sum(-1, keepdims=True)
        return e / np.where(total == 0, 1.0, total)


def route(logits, top, bias=None, mask=None, score="softmax", groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0):
    """weights and experts, [rows][top]."""
    x = np.asarray(logits, dtype=np.float64)
    rows, count = x.shape
    weights, experts = np.zeros((rows, top)), np.full((rows, top), NONE)
    b = np.zeros(count) if bias is None else np.asarray(bias, dtype=np.float64)
    size = count // groups
    for r in range(rows):
        if mask is not None and not mask[r]:
            continue
        if np.isnan(x[r]).any() or np.isnan(b).any() or (score == "softmax" and (x[r] == np.inf).any()):
            weights[r] = np.nan
            continue
        s = scores(x[r:r + 1], score)[0]
        out = (x[r] == -np.inf) | (b == -np.inf)
        scored = np.where(out, -np.inf, s + b)
        keys = np.where(out, -np.inf, x[r]) if bias is None else scored
        if groups > 1:
            best = np.full(groups, -np.inf)
            for g in range(groups):
                mine = sorted((scored if group_top > 1 else keys)[g * size:(g + 1) * size], reverse=True)[:group_top]
                mine = [v for v in mine if v > -np.inf]
                if mine:
                    best[g] = sum(mine)
            stay = sorted(range(groups), key=lambda g: (-best[g], g))[:top_groups]
            keys = np.array([keys[e] if e // size in stay else -np.inf for e in range(count)])
        order = [e for e in sorted(range(count), key=lambda e: (-keys[e], e)) if keys[e] > -np.inf][:top]
        if not order:
            continue
        experts[r, :len(order)] = order
        w = s[order]
        if renormalise:
            # ratios of the chosen scores, which may all be too small for numbers of 64 bits
            l = x[r, order]
            log = l if score == "softmax" else -np.logaddexp(0.0, -l)
            w = np.exp(log - log.max())
            w /= w.sum()
        weights[r, :len(order)] = scale * w
    return weights, experts


def route_grad(dweights, logits, experts, score="softmax", renormalise=True, scale=1.0):
    x, d = np.asarray(logits, dtype=np.float64), np.asarray(dweights, dtype=np.float64)
    rows, count = x.shape
    out = np.zeros_like(x)
    s = scores(x, score)
    for r in range(rows):
        chosen = [(j, e) for j, e in enumerate(experts[r]) if 0 <= e < count]
        if not chosen:
            continue
        # derivative of weight j with respect to each score, times the score's with respect to the logits
        ds = np.zeros(count)
        total = sum(s[r, e] for _, e in chosen)
        if renormalise:
            # q = s / total: log-derivatives, so that tiny scores are no trouble
            l = np.array([x[r, e] for _, e in chosen])
            log = l if score == "softmax" else -np.logaddexp(0.0, -l)
            q = np.exp(log - log.max())
            q /= q.sum()
            back = np.array([d[r, j] for j, _ in chosen])
            inner = q * (back - (q * back).sum()) * scale
            for (_, e), v in zip(chosen, inner):
                out[r, e] += v * (1.0 if score == "softmax" else 1.0 - s[r, e])
            continue
        for j, e in chosen:
            ds[e] += scale * d[r, j]
        if score == "sigmoid":
            out[r] = ds * s[r] * (1 - s[r])
        else:
            out[r] = s[r] * (ds - (ds * s[r]).sum())
    return out


def order(experts, count):
    flat = [e if 0 <= e < count else count for e in np.asarray(experts).reshape(-1).tolist()]
    where = [[] for _ in range(count + 1)]
    for i, e in enumerate(flat):
        where[e].append(i)
    places = np.zeros(len(flat), dtype=np.int64)
    ends, at = [], 0
    for e in range(count + 1):
        for i in where[e]:
            places[i] = at
            at += 1
        ends.append(at)
    return places.reshape(np.asarray(experts).shape), np.array(ends[:count], dtype=np.int64)


def dispatch(x, places):
    rows, top = places.shape
    out = np.zeros((rows * top, x.shape[1]))
    for r in range(rows):
        for j in range(top):
            out[places[r, j]] = x[r]
    return out


def combine(y, places, weights=None):
    rows, top = places.shape
    out = np.zeros((rows, y.shape[1]))
    for r in range(rows):
        for j in range(top):
            w = 1.0 if weights is None else weights[r, j]
            if w != 0 and 0 <= places[r, j] < rows * top:
                out[r] += w * y[places[r, j]]
    return out


def combine_grad(dout, y, places, weights):
    rows, top = places.shape
    dy, dw = np.zeros_like(y), np.zeros((rows, top))
    for r in range(rows):
        for j in range(top):
            if 0 <= places[r, j] < rows * top:
                dy[places[r, j]] = weights[r, j] * dout[r]
                dw[r, j] = (dout[r] * y[places[r, j]]).sum()
    return dy, dw


def int_scale(v):
    """fp32 scale of rows: largest magnitude / 127, 2^-126 at least; NaN for rows that are not finite."""
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(v).max(-1).astype(np.float32)
        s = np.maximum((top / np.float32(127)).astype(np.float32), np.float32(2.0 ** -126))
    return np.where(np.isfinite(v).all(-1), s, np.float32(np.nan)).astype(np.float32)


def int_quantize(x, diag=None, block=0):
    """codes [rows][k] and scales of exactly rotated rows."""
    v = rotate(x, diag, block)
    scale = int_scale(v)
    s = scale.astype(np.float64)[:, None]
    with np.errstate(invalid="ignore"):
        codes = np.where(np.isfinite(s), np.rint(v / s), 0.0)               # to the nearest, ties to even
    return np.where(np.isfinite(codes), codes, 0.0).astype(np.int64), scale


def int_products(a_codes, a_scales, w_codes, w_scales, ends=None):
    """a w^T of codes [rows][k] and [experts][n][k]: whole sums, then both scales; rows of no expert 0."""
    a, w = np.asarray(a_codes, dtype=np.int64), np.asarray(w_codes, dtype=np.int64)
    rows, experts = a.shape[0], w.shape[0]
    out, at = np.zeros((rows, w.shape[1])), 0
    for e in range(experts):
        end = rows if ends is None else max(at, min(rows, max(0, int(ends[e]))))
        if end > at:
            sums = (a[at:end].astype(np.float64) @ w[e].T.astype(np.float64))          # whole numbers below 2^53
            out[at:end] = sums * w_scales[e].astype(np.float64)[None] * a_scales[at:end].astype(np.float64)[:, None]
        at = end
    return out
