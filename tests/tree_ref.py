"""Plain float64 forms of the tree operators, used by the tests of them."""

from __future__ import annotations

import math

import numpy as np


def random_parents(n, rng, back=4):
    """Node 0 is the root; a node hangs below one of the `back` before it."""
    return np.array([-1] + [max(0, i - 1 - int(rng.integers(back))) for i in range(1, n)], np.int32)


def layout(parents):
    """Depths, and a truth table [n, n]: node i sees node j."""
    n = len(parents)
    depth, see = np.zeros(n, np.int32), np.zeros((n, n), bool)
    for i, p in enumerate(parents):
        if p >= 0:
            depth[i], see[i] = depth[p] + 1, see[p]
        see[i, i] = True
    return depth, see


def pack(see):
    """Truth table [n, m] as uint64 words, bit j % 64 of word j // 64."""
    n, m = see.shape
    out = np.zeros((n, (m + 63) // 64), np.uint64)
    for j in range(m):
        out[:, j // 64] |= see[:, j].astype(np.uint64) << np.uint64(j % 64)
    return out


def rope(x, positions, form):
    """x [n, heads, D] float64, turned; form: the keywords of binding.rope."""
    R, s = form["rotary_dim"], form.get("factor", 1.0)
    base, kind = form.get("base", 10000.0), form.get("scaling", "none")
    out, gain = x.copy(), 1.0
    for i in range(R // 2):
        f = base ** (-2.0 * i / R)
        if kind == "linear":
            f = f / s
        elif kind == "ntk":
            f = (base * s ** (R / (R - 2.0))) ** (-2.0 * i / R)
        elif kind == "yarn":
            turns = form.get("original_context", 4096) * f / (2.0 * math.pi)
            slow, fast = form.get("beta_slow", 1.0), form.get("beta_fast", 32.0)
            g = min(1.0, max(0.0, (turns - slow) / (fast - slow)))
            f = f * g + f / s * (1.0 - g)
            gain = 0.1 * math.log(s) + 1.0
        gain = form.get("gain") or gain
        a, b = (i, i + R // 2) if form.get("layout", "half") == "half" else (2 * i, 2 * i + 1)
        ang = np.asarray(positions, np.float64) * f
        c, d = gain * np.cos(ang)[:, None], gain * np.sin(ang)[:, None]
        out[:, :, a] = x[:, :, a] * c - x[:, :, b] * d
        out[:, :, b] = x[:, :, b] * c + x[:, :, a] * d
    return out


def attention(q, k, v, prefix, see, scale):
    """q [n, H, D], k and v [KVH, positions, D], see [n, n]; float64.  Keys and
    values that a row does not see are left out.  Also the largest sum of
    |q_e k_e scale| of a row's visible keys (for tolerances)."""
    n, H, D = q.shape
    G = H // k.shape[0]
    out, size = np.zeros((n, H, D)), 0.0
    for r in range(n):
        cols = np.concatenate([np.arange(prefix), prefix + np.nonzero(see[r])[0]]).astype(int)
        if not len(cols):
            continue
        for h in range(H):
            kk, vv = k[h // G, cols], v[h // G, cols]
            s = kk @ q[r, h] * scale
            size = max(size, float((np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)))
            p = np.exp(s - s.max())
            out[r, h] = p @ vv / p.sum()
    return out, size


def attention_tol(D, keys, size, vmax):
    """Error of a float32 evaluation with exact products: four standard
    deviations of the roundings (2^-24 each) of a score of 3 D terms, whose
    absolute value is at most size, and of sums over 3 keys terms."""
    return 2.0 ** -24 * (4 * math.sqrt(3 * D + 8) * size + 4 * math.sqrt(3 * keys) + 16) * vmax


def walk(logits, tokens, parents):
    """[count, next, path, -1 .., best]: the greedy walk."""
    n = len(tokens)
    x = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    best = x.argmax(axis=1)
    best[np.isnan(logits).all(axis=1)] = 0
    # an all -inf row's numbers all tie; a NaN among them does not win
    for r in range(n):
        if np.isneginf(x[r]).all() and not np.isnan(logits[r]).all():
            best[r] = int(np.nonzero(~np.isnan(logits[r]))[0][0])
    path, cur = [0], 0
    while True:
        kids = [i for i in range(cur + 1, n) if parents[i] == cur and tokens[i] == best[cur]]
        if not kids:
            break
        cur = kids[0]
        path.append(cur)
    return np.array([len(path), best[cur]] + path + [-1] * (n - len(path)) + list(best), np.int32)


def keep(kv, base, path):
    """kv [planes, capacity, D] with the rows of the path moved together."""
    out = kv.copy()
    for i, p in enumerate(path):
        out[:, base + i] = kv[:, base + p]
    return out
