"""Plain definitions, in 64 bits, of a cache in 8 bits (e4m3 with a power of two for each block of
rows and head), of the pages of sequences that go on or fork, and of the verification of drafted
tokens.  Nothing here is shared with the GPU path."""
from __future__ import annotations

import math

import numpy as np

RANGE = {"f16": (-15, 7), "bf16": (-117, 119)}


def e4m3(b):
    """The values of e4m3 bytes: sign, 4 bits of exponent (bias 7), 3 of mantissa, no infinities."""
    b = np.asarray(b, np.uint8).astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    x = np.where((b & 127) == 127, np.nan, x)
    return np.where(b >> 7 == 1, -x, x)


_FINITE = np.array([float(e4m3(b)) for b in range(127)])        # ascending


def to_e4m3(x):
    """Bytes of the nearest values (ties to the even mantissa, at most 448); NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.minimum(np.abs(x), 448.0), 0.0)
    hi = np.searchsorted(_FINITE, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _FINITE[hi] - a, a - _FINITE[lo]
    b = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    b = np.where(np.isfinite(x), b, 127)
    return (b + 128 * np.signbit(x)).astype(np.uint8)


def exponent(x, dtype):
    """The least exponent with which the finite values of x are at most 448, in the type's range."""
    lo, hi = RANGE[dtype]
    x = np.abs(np.asarray(x, np.float64))
    top = np.max(x[np.isfinite(x)], initial=0.0)
    for e in range(lo, hi):
        if top <= 448.0 * 2.0 ** e:
            return e
    return hi


def append(k8, v8, ex, row_of, lens, key, value, block, dtype, counts=None, room=10 ** 9):
    """k8, v8 (pages, page, heads, d) bytes and ex (pages, blocks, heads, 2), changed in place; row_of(b,
    n) as oracle.cache.row_of; key, value (sequences, tokens, heads, d) values of the 16-bit type."""
    B, T, heads, _ = key.shape
    for b in range(B):
        n0 = min(max(int(lens[b]), 0), room)
        t = T if counts is None else min(max(int(counts[b]), 0), T)
        end = min(n0 + t, room)
        for begin in range(n0 // block * block, end, block):
            r = row_of(b, begin)
            if r is None:
                continue
            p, s = r
            old, new = max(n0 - begin, 0), min(begin + block, end) - begin
            if new <= old:      # nothing is appended
                continue
            for h in range(heads):
                for i, (pool, x) in enumerate(((k8, key), (v8, value))):
                    rows = x[b, begin + old - n0:begin + new - n0, h]
                    e = exponent(rows, dtype)
                    was = max(int(ex[p, s // block, h, i]), -126)
                    if old and was >= e:
                        e = was
                    elif old:
                        y = e4m3(pool[p, s:s + old, h]) * 2.0 ** (was - e)
                        pool[p, s:s + old, h] = to_e4m3(y)
                    pool[p, s + old:s + new, h] = to_e4m3(rows * 2.0 ** -e)
                    ex[p, s // block, h, i] = e


def pages(table, lens, tokens, pages, page, parent=None):
    """(table, lengths, copies, lacking) of the sequences that continue their parents."""
    B, width = table.shape
    heirs = list(range(B)) if parent is None else [int(p) if 0 <= p < B else -1 for p in parent]
    room = width * page
    n = [min(max(int(lens[p]), 0), room) if p >= 0 else 0 for p in heirs]
    row = [table[p] if p >= 0 else np.full(width, -1) for p in heirs]
    real = lambda x: 0 <= x < pages                                          # noqa: E731
    held = {int(x) for i in range(len(heirs)) for x in row[i][:n[i] // page] if real(x)}
    keeper = {}
    for i in range(len(heirs)):
        if n[i] % page and real(row[i][n[i] // page]):
            x = int(row[i][n[i] // page])
            if x not in held:
                keeper.setdefault(x, i)
    free = (x for x in range(pages) if x not in held and x not in keeper)
    out = np.full((len(heirs), width), -1, np.int32)
    copies = np.tile(np.array([-1, -1, 0], np.int32), (len(heirs), 1))
    lacking = np.zeros(len(heirs), np.int32)

    def take(i):
        x = next(free, -1)
        lacking[i] += x < 0
        return x
    for i in range(len(heirs)):
        have = -(-n[i] // page)
        out[i, :have] = row[i][:have]
        if n[i] % page:
            x = int(row[i][have - 1])
            if real(x) and keeper.get(x) != i:
                out[i, have - 1] = take(i)
                if out[i, have - 1] >= 0:
                    copies[i] = x, out[i, have - 1], n[i] % page
        for w in range(have, -(-min(n[i] + tokens, room) // page)):
            out[i, w] = take(i)
    return out, np.array(n, np.int32), copies, lacking


def verify(tokens, target, uniform, draft=None, parent=None, counts=None):
    """(path, found, next) for target (sequences, nodes, vocabulary), by the rule's words."""
    def clean(x):
        x = np.asarray(x, np.float64)
        return np.where((x > 0) & np.isfinite(x), x, 0.0)
    B, T, V = target.shape
    path, found = np.full((B, T), -1, np.int32), np.zeros(B, np.int32)
    nxt = np.full(B, -1, np.int64)
    for b in range(B):
        size = T if counts is None else min(max(int(counts[b]), 0), T)
        if size == 0:
            continue
        up = list(range(-1, T - 1)) if parent is None else [int(x) for x in
                                                            (parent if parent.ndim == 1 else parent[b])]
        u = [min(max(float(x), 0.0), 1.0 - 2.0 ** -24) for x in uniform[b]]
        c, way, refused, gone = 0, [0], False, []
        p = clean(target[b, 0])
        at = lambda r, x: r[x] if 0 <= x < V else 0.0                        # noqa: E731
        for n in range(1, size):
            if not 0 <= up[n] < n or up[n] != c:
                continue
            x = int(tokens[b, n])
            if draft is not None:
                yes = u[n] * at(clean(draft[b, c]), x) < at(p, x)
                refused = not yes
            else:
                left = 1.0 - math.fsum(at(p, y) for y in set(gone))
                yes = x not in gone and at(p, x) > 0 and u[n] * left < at(p, x)
                if not yes:
                    gone.append(x)
            if yes:
                c, gone = n, []
                way.append(n)
                p = clean(target[b, c])
        r = p.copy()
        if refused:
            r = np.maximum(p - clean(draft[b, c]), 0.0)
        for y in gone:
            if 0 <= y < V:
                r[y] = 0.0
        if not r.any():
            r = p
        path[b, :len(way)], found[b] = way, len(way)
        if r.any():
            sums = np.cumsum(r)
            nxt[b] = min(int(np.searchsorted(sums, u[0] * sums[-1], side="right")),
                         int(np.flatnonzero(r)[-1]))
    return path, found, nxt
