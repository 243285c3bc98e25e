"""Calls of paged_attention by how they are shared out, and their plain float64 form a
sequence at a time, for the tests of calls that are too large for the other's loops."""

from __future__ import annotations

import collections
import ctypes
import math

import numpy as np

from paper_2309_08168_amd import binding
from tests import paged_ref as P
from tests import tree_ref as T

Plan = collections.namedtuple("Plan", "tile slots chunks span splits waves wide")
Call = collections.namedtuple("Call", "rows lengths heads kvh page max_rows")

# a weight of a bfloat16 call is one bfloat16 term, or two where a kv head has few rows; over float32
# pages it is not rounded
WEIGHT = {"one": 2.0 ** -8, "two": 2.0 ** -16, "float32": 0.0}


def width(c):
    """Pages of a row of the table (as Cache of the GPU tests has them)."""
    return max([-(-n // c.page) for n in c.lengths] + [1]) + 1


def plan(kv, batch, x, heads, n):
    out = (ctypes.c_int32 * 7)()
    binding.check(binding.load().sdk_paged_plan(ctypes.byref(kv), ctypes.byref(batch), int(x == "bf16"), heads, n, out))
    return Plan(*out)


def plan_of(c, d, x, dtype, max_length=0):
    """The plan of a call, without its tensors (nothing reads the addresses)."""
    at, step = 1 << 20, d * c.page
    kv = binding.sd_kv_pages(at, at, step * c.kvh, step, d, c.kvh, 1 << 20, c.page, d, int(dtype == "bf16"))
    batch = binding.sd_batch(at, at, at, width(c), len(c.lengths), width(c), c.max_rows, max_length)
    return plan(kv, batch, x, c.heads, sum(c.rows))


def layout(c, p):
    """Of the streams of a call the sequences of each chunk: [(sequence, its first span there, its end, its spans), ...]."""
    spans = [max(1, -(-n // p.span)) if m else 0 for m, n in zip(c.rows, c.lengths)]
    before = np.concatenate([[0], np.cumsum(spans)])
    step = max(1, -(-int(before[-1]) // p.chunks))
    chunks = []
    for k in range(p.chunks):
        lo, hi = k * step, min((k + 1) * step, int(before[-1]))
        chunks.append([(s, max(lo, b) - b, min(hi, b + m) - b, m) for s, (b, m) in enumerate(zip(before, spans))
                       if m and max(lo, b) < min(hi, b + m)])
    return chunks, step


def parts(c, p):
    """Most chunks that a sequence is in."""
    return max(collections.Counter(t[0] for k in layout(c, p)[0] for t in k).values())


def attention(q, k, v, length, rows, limit, scale, there=None):
    """Rows (m of them, the first `rows` taken) of a sequence over its positions: q [m, G, d], k and v [length, d] of a kv head,
    there [length]: whether a position has a page.  (output, largest sum of |q_e k_e scale|, weighted mean of |v|)."""
    m, G, d = q.shape
    see = np.arange(length)[None, :] <= (length - m + np.arange(rows))[:, None]
    see &= (np.arange(length) < limit)[None, :]
    if there is not None:
        see &= there[None, :]
    see = np.repeat(see, G, axis=0)
    x = q[:rows].reshape(rows * G, d)
    z = np.where(see, x @ k.T * scale, -np.inf)
    top = np.where(see.any(axis=1), z.max(axis=1, initial=-np.inf), 0.0)
    w = np.exp(z - top[:, None])
    w /= np.maximum(w.sum(axis=1, keepdims=True), 1e-300)
    size = float((np.abs(x) @ np.abs(k).T).max(initial=0.0) * abs(scale))
    return (w @ v).reshape(rows, G, d), size, (w @ np.abs(v)).reshape(rows, G, d)


def tolerance(x, weight, d, keys, size, vmax, want, spread):
    """Float32 sums (the helper of the tree operators), the weights' rounding and, of bfloat16 results, theirs."""
    tol = T.attention_tol(d, keys, size, vmax) + (WEIGHT[weight] * spread if x == "bf16" else 0.0)
    return tol * (1 + P.HALF[x]) + P.HALF[x] * np.abs(want) if x == "bf16" else tol


def weight_of(p, dtype):
    return "float32" if dtype == "f32" else "two" if p.tile <= 32 else "one"


def scale_of(d):
    return 1.0 / math.sqrt(d)


# ----------------------------------------------------------------------------
# Streams whose chunks have several spans: chunks that hold several sequences, ones that end one
# sequence and begin another, sequences of many parts; empty ones between.  By the rows of a tile
# and the waves of a work-group.

LONG, SHORT = [0, 40, 3000, 1, 130, 2437, 177, 355], [0, 40, 1500, 1, 130, 347, 781, 1125]
STREAMS = {
    # (tile, waves): Call
    (16, 4): Call([1, 1, 1, 1, 0, 1, 1, 1], SHORT, 64, 32, 32, 1),
    (16, 8): Call([1, 3, 4, 1, 0, 2, 4, 1], LONG, 128, 32, 64, 4),
    (32, 4): Call([2, 4, 3, 1, 0, 4, 1, 4], LONG, 256, 32, 16, 4),
    (64, 4): Call([8, 1, 7, 1, 0, 8, 3, 5], LONG, 256, 32, 64, 8),
    (128, 4): Call([13, 2, 16, 1, 0, 16, 9, 5], LONG, 256, 32, 32, 16),
}

# Sequences of more parts than a wave has lanes: (tile, threads of the join): Call.  (Eight waves
# have spans of 256 keys: 79 of 20000.)
MANY_PARTS = {
    (16, 256): Call([3], [20000], 4, 1, 128, 3),
    (16, 64): Call([2] * 20 + [4] + [1] * 19, list(range(30, 50)) + [20000] + [3] * 10 + [600] * 9, 4, 1, 128, 4),
    (32, 256): Call([4, 1], [20000, 5], 8, 1, 64, 4),
    (64, 256): Call([1, 8], [300, 20000], 8, 1, 64, 8),
    (128, 256): Call([2, 16], [300, 20000], 8, 1, 32, 16),
    (128, 64): Call([16] + [1] * 70, [9000] + [70] * 70, 8, 1, 32, 16),
}


# Around as many sequences as a work-group of a stream adds up the spans of (1024), several hundred of
# more than one span, by (sequences, rows of a tile): two or four sequences a thread.
def many_sequences(n, tile):
    rng = np.random.default_rng(n + tile)
    most = {16: 1, 32: 3, 64: 8, 128: 16}[tile]
    heads = 2 if tile == 16 else 8
    lengths = [int(t) for t in rng.integers(0, 700, n)]
    lengths[n // 3], lengths[n - 1] = 2100, 1500
    rows = [int(t) for t in rng.integers(0, most + 1, n)]
    rows[0], rows[n - 1] = most, 1
    return Call(rows, lengths, heads, 1, 64, most)


MANY = [(n, tile) for n in (513, 1023, 1024, 1025) for tile in (16, 32, 64, 128)]

# Tiles over pages, whole and in shares, of few and of many sequences.
CHUNKS, BEHIND = [200, 1, 130, 90, 64], [700, 300, 130, 500, 1000]
_rng = np.random.default_rng(70)
SEVENTY = [int(t) for t in _rng.integers(0, 71, 70)]
SEVENTY[5] = 70
AFTER = [m + int(t) for m, t in zip(SEVENTY, _rng.integers(0, 500, 70))]
TILES = {
    # (name, type of the queries): (Call, tile, shares or 0: more than one, whether by k_batch_attn_wide)
    ("five chunks, 64-row tiles", "f32"): (Call(CHUNKS, BEHIND, 64, 32, 64, 200), 64, 1, 0),
    ("five chunks, 64-row tiles", "bf16"): (Call(CHUNKS, BEHIND, 64, 32, 16, 200), 64, 1, 0),
    ("five chunks, tiles for every CU", "f32"): (Call(CHUNKS, BEHIND, 80, 40, 16, 200), 128, 1, 0),
    ("five chunks, tiles for every CU", "bf16"): (Call(CHUNKS, BEHIND, 80, 40, 64, 200), 128, 1, 1),
    ("five chunks, small pages", "bf16"): (Call(CHUNKS, BEHIND, 80, 40, 16, 190), 128, 1, 1),
    ("one chunk", "f32"): (Call([700], [1111], 64, 32, 32, 700), 64, 1, 0),
    ("one chunk", "bf16"): (Call([700], [1111], 64, 32, 32, 700), 128, 1, 1),
    ("one chunk, no past", "bf16"): (Call([700], [700], 64, 32, 128, 700), 128, 1, 1),
    ("70 sequences, shares", "f32"): (Call(SEVENTY, AFTER, 4, 2, 64, 70), 128, 0, 0),
    ("70 sequences, shares", "bf16"): (Call(SEVENTY, AFTER, 4, 2, 16, 70), 128, 0, 1),
    ("70 sequences, 64-row tiles", "f32"): (Call(SEVENTY, AFTER, 8, 4, 16, 70), 64, 1, 0),
    ("70 sequences, 64-row tiles", "bf16"): (Call(SEVENTY, AFTER, 8, 4, 64, 70), 64, 1, 0),
    ("70 sequences, tiles for every CU", "f32"): (Call(SEVENTY, AFTER, 12, 6, 64, 70), 128, 1, 0),
    ("70 sequences, tiles for every CU", "bf16"): (Call(SEVENTY, AFTER, 12, 6, 32, 69), 128, 1, 1),
}

# Up to 32 rows of a kv head without streams, by (rows of a tile, waves): Call.
FEW = {
    (16, 4): Call([1, 3, 2, 4, 0, 1], [300, 40, 333, 64, 7, 1], 16, 4, 32, 4),
    (32, 4): Call([5, 8, 1, 7], [250, 33, 410, 7], 16, 4, 16, 8),
    (16, 1): Call([1, 2, 0, 2] * 4, [100, 33, 5, 200] * 4, 344, 43, 16, 2),
    (32, 1): Call([4, 2, 3, 1] * 4, [100, 33, 5, 401] * 4, 344, 43, 16, 4),
}
