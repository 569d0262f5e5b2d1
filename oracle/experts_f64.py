"""Float64 definitions of a layer of experts and of the update of its tensors: routing,
rows to the experts and back, products grouped by expert, AdamW's moments in 8 bits.

Plain NumPy, test infrastructure only; nothing here is used by the library.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256  # values of a moment that share a scale


# ------------------------------------------------------------------- routing
def choose(logits, top_k: int):
    """[tokens, top_k] experts, largest logit first, lower index first among equals; -1 where none
    is left.  -inf and NaN are never chosen."""
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    order = np.argsort(-x, axis=-1, kind="stable")[:, :top_k]
    return np.where(np.take_along_axis(x, order, -1) == -np.inf, -1, order).astype(np.int64)


def probabilities(logits, expert, over: str):
    """[tokens, experts]: the softmax that weights come from, 0 where nothing has a part."""
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    if over == "chosen":
        kept = np.zeros(x.shape, bool)
        for c in range(expert.shape[1]):
            live = expert[:, c] >= 0
            kept[np.nonzero(live)[0], expert[live, c]] = True
        x = np.where(kept, x, -np.inf)
    top = x.max(-1, keepdims=True)
    with np.errstate(invalid="ignore"):
        e = np.where(x == top, 1.0, np.exp(x - top))
    e = np.where(x == -np.inf, 0.0, e)
    total = e.sum(-1, keepdims=True)
    return np.divide(e, total, out=np.zeros_like(e), where=total > 0)


def weights(logits, expert, over: str):
    p = probabilities(logits, expert, over)
    return np.where(expert >= 0, np.take_along_axis(p, np.maximum(expert, 0), -1), 0.0)


def plan(expert, experts: int):
    """(row [tokens, top_k], offset [experts + 1]): choices sorted by expert, then by token."""
    row = np.full(expert.shape, -1, np.int64)
    offset = np.zeros(experts + 1, np.int64)
    at = 0
    for e in range(experts):
        offset[e] = at
        for t, c in np.argwhere(expert == e):
            row[t, c] = at
            at += 1
    offset[experts] = at
    return row, offset


def route_backward(logits, expert, dweight, over: str):
    p = probabilities(logits, expert, over)
    d = np.zeros_like(p)
    for c in range(expert.shape[1]):
        live = expert[:, c] >= 0
        d[np.nonzero(live)[0], expert[live, c]] += np.asarray(dweight, np.float64)[live, c]
    return p * (d - (p * d).sum(-1, keepdims=True))


# ---------------------------------------------------------------------- rows
def dispatch(x, row, rows):
    """rows with rows[row[t, c]] = x[t]."""
    out = np.array(rows, np.float64)
    for t, c in np.argwhere(row >= 0):
        out[row[t, c]] = x[t]
    return out


def combine(rows, row, weight):
    """y[t] = sum over c of weight[t, c] rows[row[t, c]]."""
    y = np.zeros((row.shape[0], rows.shape[1]))
    for t, c in np.argwhere(row >= 0):
        y[t] += weight[t, c] * rows[row[t, c]]
    return y


def combine_backward(rows, dy, row, weight, drows):
    out, dweight = np.array(drows, np.float64), np.zeros(weight.shape)
    for t, c in np.argwhere(row >= 0):
        out[row[t, c]] = weight[t, c] * dy[t]
        dweight[t, c] = dy[t] @ rows[row[t, c]]
    return out, dweight


# ------------------------------------------------------------------ products
def gelu(z):
    return z * 0.5 * (1.0 + np.vectorize(math.erf, otypes=[float])(z / math.sqrt(2.0)))


def gelu_slope(z):
    return (0.5 * (1.0 + np.vectorize(math.erf, otypes=[float])(z / math.sqrt(2.0)))
            + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi))


def by_group(form: str, a, b, offset):
    """The product of every group: rows of a (xwt, xw: [rows, .], 0 for rows of no group) or one
    matrix a group (xtw)."""
    groups = len(offset) - 1
    if form == "xtw":
        return np.stack([a[offset[g]:offset[g + 1]].T @ b[offset[g]:offset[g + 1]] for g in range(groups)])
    out = np.zeros((a.shape[0], b.shape[1] if form == "xwt" else b.shape[2]))
    for g in range(groups):
        out[offset[g]:offset[g + 1]] = a[offset[g]:offset[g + 1]] @ (b[g].T if form == "xwt" else b[g])
    return out


# --------------------------------------------------------- moments in 8 bits
def e4m3_values():
    """Of the 256 codes of the format with four bits of exponent (bias 7) and three of fraction."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((e == 15) & (f == 7), np.nan, v)
    return np.where(c >> 7, -v, v)


def root_values():
    """Code c > 0 is (1 + (c % 16) / 16) 2^(floor(c / 16) - 16), code 0 is 0."""
    c = np.arange(256)
    return np.where(c > 0, (1 + (c % 16) / 16.0) * 2.0 ** (c // 16 - 16.0), 0.0)


def decode(codes, scales, values):
    """A tensor's values; the last block may be short."""
    codes = np.asarray(codes).astype(np.int64)
    with np.errstate(invalid="ignore"):  # the scale of a block that is not finite
        return values[codes] * np.repeat(np.asarray(scales, np.float64), BLOCK)[:codes.size]
