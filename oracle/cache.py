"""Plain definitions, in 64 bits, of the calls on a cache of key and value rows:
rotary positions, appended rows, attention with its weights, and eviction.
Rows are held as float64 arrays; nothing here is shared with the GPU path."""
from __future__ import annotations

import numpy as np


def frequencies(rot, base=10000.0, linear=1.0, ramp=None):
    """Radians a position of every pair."""
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)]) / linear
    if ramp is not None:
        s, length, low, high = ramp
        g = np.clip((length * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        f = f / s * (1 - g) + f * g
    return f


def rotary(x, pos, freq, layout="half", factor=1.0, inverse=False):
    """x (..., heads, d), pos (...): every pair (a, b) becomes factor (a cos - b
    sin, b cos + a sin) of pos * freq (transposed where inverse)."""
    y = np.array(x, np.float64)
    angle = np.asarray(pos, np.float64)[..., None] * freq
    if inverse:
        angle = -angle
    c, s = factor * np.cos(angle)[..., None, :], factor * np.sin(angle)[..., None, :]
    p = len(freq)
    if layout == "half":
        ia, ib = slice(0, p), slice(p, 2 * p)
    else:
        ia, ib = slice(0, 2 * p, 2), slice(1, 2 * p, 2)
    a, b = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def row_of(table, page, pages, b, n):
    """(page, slot) of row n of sequence b, or None where it does not exist."""
    w = n // page
    if table is None:
        p = b if w == 0 else -1
    else:
        p = int(table[b, w]) if w < table.shape[1] else -1
    return (p, n % page) if 0 <= p < pages else None


def visible(length, tokens, tree_row, u):
    """Rows that token u sees: all before `length`, and of the tokens' own
    those in its mask (tree_row: words, or None for a chain)."""
    own = [w for w in range(tokens)
           if (w <= u if tree_row is None else (int(tree_row[w // 64]) >> (w % 64)) & 1)]
    return list(range(length)) + [length + w for w in own]


def attend(k, v, table, lengths, q, tree, scale, counts=None):
    """k, v (pages, page, heads, d), q (sequences, tokens, query heads, d), tree
    (sequences, tokens, words) uint64 or None.  Returns out, lse, weight (sequences, heads,
    room), and for error bounds sum p |v| and max_n scale sum |q_i k_ni| per row."""
    pages, page, heads, d = k.shape
    B, T, q_heads, _ = q.shape
    group = q_heads // heads
    room = page if table is None else table.shape[1] * page
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, dots = np.full((B, T, q_heads), -np.inf), np.zeros((B, T, q_heads))
    weight = np.zeros((B, heads, room))
    for b in range(B):
        n0 = min(max(int(lengths[b]), 0), room)
        t = T if counts is None else min(max(int(counts[b]), 0), T)
        for u in range(t):
            rows = [(n, row_of(table, page, pages, b, n))
                    for n in visible(n0, t, None if tree is None else tree[b, u], u) if n < room]
            rows = [(n, r) for n, r in rows if r is not None]
            if not rows:
                continue
            n, p, s = (np.array(x) for x in zip(*[(n, r[0], r[1]) for n, r in rows]))
            for i in range(q_heads):
                kk, vv = k[p, s, i // group], v[p, s, i // group]
                x = scale * (kk @ q[b, u, i])
                dots[b, u, i] = np.max(abs(scale) * (np.abs(kk) @ np.abs(q[b, u, i])))
                top = x.max()
                e = np.exp(x - top)
                lse[b, u, i] = top + np.log(e.sum())
                e /= e.sum()
                out[b, u, i], mag[b, u, i] = e @ vv, e @ np.abs(vv)
                weight[b, i // group, n] += e
    return out, lse, weight, mag, dots


def evict(weight, n, keep, sink, recent):
    """The kept rows of one sequence of n rows, ascending."""
    if n <= keep:
        return np.arange(n)
    w = np.zeros(n)
    m = min(n, len(weight))
    w[:m] = weight[:m]
    w = np.where(np.isnan(w), -np.inf, w) + 0.0
    mid = sorted(range(sink, n - recent), key=lambda i: (-w[i], i))
    return np.array(sorted(list(range(sink)) + mid[:keep - sink - recent]
                           + list(range(n - recent, n))), np.int64)
