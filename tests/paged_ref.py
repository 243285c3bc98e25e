"""Plain float64 forms of the operators of batches, used by the tests of them."""

from __future__ import annotations

import numpy as np

from tests import tree_ref as T

# half a step of a rounding, relative to the value
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def row_places(starts, lengths, n, max_rows):
    """Of each packed row (sequence, position), or None where no sequence takes it."""
    out = [None] * n
    for s in range(len(lengths)):
        m = starts[s + 1] - starts[s]
        for i in range(min(m, max_rows)):
            out[starts[s] + i] = (s, lengths[s] - m + i)
    return out


def page_row(table, s, p, page, n_pages, max_length):
    """(page, row of it) of a position, or None where it has no place."""
    if not 0 <= p < max_length or p // page >= table.shape[1]:
        return None
    b = int(table[s, p // page])
    return (b, p % page) if 0 <= b < n_pages else None


def normed(x, weight, eps):
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * weight


def attention(q, keys, values, seen, scale):
    """q [n, H, D]; keys and values: a function of a row and a kv head giving those it
    sees, [k, D]; seen(row): whether the row is one of a sequence.  Returns the output
    (NaN for rows of none), the largest sum of |q_e k_e scale|, and per row and head
    the weighted mean of |v|, [n, H, D]."""
    n, H, D = q.shape
    out, spread, size = np.full((n, H, D), np.nan), np.zeros((n, H, D)), 0.0
    for r in range(n):
        if not seen(r):
            continue
        for h in range(H):
            kk, vv = keys(r, h), values(r, h)
            if not len(kk):
                out[r, h] = 0.0
                continue
            s = kk @ q[r, h] * scale
            size = max(size, float((np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)))
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h], spread[r, h] = p @ vv, p @ np.abs(vv)
    return out, size, spread


def attention_tol(x, D, keys, size, vmax, want, spread):
    """Float32 sums (the helper of the tree operators); bfloat16 queries also round
    the softmax weights, each by half a step of itself, and the result."""
    tol = T.attention_tol(D, keys, size, vmax)
    if x == "bf16":
        return tol * (1 + HALF[x]) + HALF[x] * (np.abs(want) + spread * (1 + HALF[x]))
    return tol

