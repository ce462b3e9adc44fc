"""Oracle of positions, norms and drafted tokens: one head, token and key at a time in fp64.

TEST INFRASTRUCTURE. Only the test-suite uses this module; the library never
imports it. The paper has no counterpart.
"""
from __future__ import annotations

import numpy as np

from .kvcache import DEVERR_PAGE, DEVERR_ROW_INDEX, DEVERR_SHARED, Cache


def rotate(x, w, eps, inv_freq, interleaved, amplitude, pos):
    """One head x [D] at position pos: the head, and the size that rounding errors are measured by."""
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt(np.mean(x * x) + eps) * np.asarray(w, np.float64)
    y, size, R = x.copy(), np.abs(x), 2 * len(inv_freq)
    for i, f in enumerate(inv_freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        cos, sin = np.cos(pos * f), np.sin(pos * f)
        y[a], y[b] = amplitude * (x[a] * cos - x[b] * sin), amplitude * (x[b] * cos + x[a] * sin)
        size[a] = size[b] = abs(amplitude) * np.hypot(x[a], x[b])
    return y, size


def masks(parent, count):
    """parent [n]: whether drafted token i < count sees j, and its depth; parents out of range count as -1."""
    n, bad = len(parent), False
    sees, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
    for i in range(count):
        j = i
        while j >= 0:
            sees[i, j] = True
            up = parent[j]
            if not -1 <= up < j:
                up, bad = -1, True
            depth[i] += up >= 0
            j = up
    return sees, depth, bad


def words(sees):
    """[n][n] truth values as [n][ceil(n / 32)] 32-bit words."""
    n = len(sees)
    out = np.zeros((n, -(-n // 32)), np.int64)
    for i, j in np.argwhere(sees):
        out[i, j // 32] |= 1 << (j % 32)
    return out.astype(np.uint32).view(np.int32)


def append_places(cache: Cache, n_new, count=None):
    """(sequence, row, token, page or None) of every row that rps_kv_append takes."""
    for s in range(len(cache.length)):
        m = n_new if count is None else max(0, min(n_new, int(count[s])))
        n = int(cache.length[s])
        if n < 0:
            continue
        if cache.pages(n) > cache.table.shape[1]:
            n = cache.table.shape[1] * cache.ps
            if m:
                cache.err |= DEVERR_PAGE
        for i in range(m):
            pos = n - m + i
            if pos < 0:
                continue
            p = int(cache.table[s, pos // cache.ps])
            if not 0 <= p < len(cache.ref):
                cache.err |= DEVERR_PAGE
                p = None
            elif cache.ref[p] > 1:
                cache.err |= DEVERR_SHARED
                p = None
            yield s, i, pos, p


def keep_path(cache: Cache, path, n_keep, n_q, count=None):
    """Moves the kept tokens of every sequence; returns the new lengths."""
    new_len = []
    for s in range(len(cache.length)):
        n = int(cache.length[s])
        if n < 0:
            new_len.append(-1)
            continue
        m = n_q if count is None else max(0, min(n_q, int(count[s])))
        keep, ctx = int(n_keep[s]), n - m
        p = [int(x) for x in path[s][:max(0, keep)]]
        if not 0 <= keep <= min(len(path[s]), m) or ctx < 0 or any(not 0 <= x < m for x in p) or any(
                a >= b for a, b in zip(p, p[1:])):
            cache.err |= DEVERR_ROW_INDEX
            new_len.append(n)
            continue
        for d, x in enumerate(p):
            if d == x:
                continue
            a, b = (int(cache.table[s, (ctx + y) // cache.ps]) for y in (x, d))
            if not (0 <= a < len(cache.ref) and 0 <= b < len(cache.ref)):
                cache.err |= DEVERR_PAGE
            elif cache.ref[b] > 1:
                cache.err |= DEVERR_SHARED
            else:
                for t in (cache.k, cache.v):
                    t[:, b, :, (ctx + d) % cache.ps] = t[:, a, :, (ctx + x) % cache.ps]
        new_len.append(ctx + keep)
    return np.array(new_len)


def tree_attention(q, cache: Cache, layer, scale, count=None, sees=None):
    """q [n_seq][n_q][H][D] (fp64): query i < m of a sequence of n tokens sees tokens j < n - m, and n - m + t where
    sees[s][i][t] (None: t <= i). out like q, the same weights over |v|, lse [n_seq][n_q][H]; what is not written: NaN."""
    n_seq, n_q, H, D = q.shape
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse = np.full((n_seq, n_q, H), np.nan)
    group = H // cache.k.shape[2]
    for s in range(n_seq):
        n = int(cache.length[s])
        if n < 0:
            continue
        m = n_q if count is None else max(0, min(n_q, int(count[s])))
        k, v = cache.rows(layer, s)
        t = np.arange(n) - (n - m)
        for i in range(m):
            seen = (t < 0) | (t <= i if sees is None else np.array([x >= 0 and bool(sees[s][i][x]) for x in t], bool))
            for h in range(H):
                z = scale * (k[seen, h // group] @ q[s, i, h])
                top = z.max() if seen.any() else -np.inf
                if top == -np.inf:
                    out[s, i, h], mag[s, i, h], lse[s, i, h] = 0.0, 0.0, -np.inf
                    continue
                p = np.exp(z - top)
                out[s, i, h] = p @ v[seen, h // group] / p.sum()
                mag[s, i, h] = p @ np.abs(v[seen, h // group]) / p.sum()
                lse[s, i, h] = top + np.log(p.sum())
    return out, mag, lse
