"""Oracle of the paged K/V cache: bookkeeping, page data and the attention that
reads it, one sequence, page and token at a time.

TEST INFRASTRUCTURE. Only the test-suite uses this module; the library never
imports it. The paper has no counterpart: a denoiser that decodes block by
block keeps the context's keys and values, and the branches of a lookahead step
(Sec. 3.1 "Lookahead scoring") share them.

State: ref [n_pages], table [n_seq][width], length [n_seq] (-1 absent), and the
data k, v [layers][pages][heads][page size][head dim] in any dtype.
"""
from __future__ import annotations

import numpy as np

DEVERR_ROW_INDEX, DEVERR_PAGE, DEVERR_NO_PAGES, DEVERR_SHARED = 0x1, 0x40, 0x80, 0x100


class Cache:
    def __init__(self, ref, table, length, page_size, k=None, v=None):
        self.ref, self.table, self.length = (np.array(x, dtype=np.int64) for x in (ref, table, length))
        self.ps, self.k, self.v, self.err = page_size, k, v, 0

    def pages(self, n: int) -> int:
        return 0 if n <= 0 else -(-n // self.ps)

    def free(self):
        return [p for p in range(len(self.ref)) if self.ref[p] <= 0]

    def _take(self, p, step):
        if 0 <= p < len(self.ref):
            self.ref[p] += step
        else:
            self.err |= DEVERR_PAGE

    def reorder(self, src, keep=None):
        table, length = self.table.copy(), self.length.copy()
        for s in range(len(length)):
            for p in table[s, : self.pages(length[s])]:
                self._take(p, -1)
        for s, f in enumerate(src):
            cut = np.iinfo(np.int64).max if keep is None else keep[s]
            if not -1 <= f < len(length):
                self.err |= DEVERR_ROW_INDEX
                f, cut = s, np.iinfo(np.int64).max
            n = -1 if f < 0 else length[f]
            n = max(-1, min(n, cut))
            m = self.pages(n)
            self.length[s] = n
            self.table[s] = -1
            self.table[s, :m] = table[f, :m]
            for p in self.table[s, :m]:
                self._take(p, 1)

    def fork_branches(self, n_branch, valid, ctx_len=None):
        src, keep = [], []
        for q in range(len(self.length) // n_branch):
            src += [q * n_branch] + [q * n_branch if valid[q][b] else -1 for b in range(n_branch - 1)]
            cut = np.iinfo(np.int64).max if ctx_len is None else ctx_len[q]
            keep += [np.iinfo(np.int64).max] + [cut] * (n_branch - 1)
        self.reorder(src, keep)

    def commit(self, n_branch, winner):
        src = []
        for q, w in enumerate(winner):
            if w >= n_branch - 1:
                self.err |= DEVERR_ROW_INDEX
                w = -1
            src += [q * n_branch + (w + 1 if w >= 0 else 0)] + [-1] * (n_branch - 1)
        self.reorder(src)

    def resize(self, new_len):
        width = self.table.shape[1]
        want = []
        for s, n in enumerate(new_len):
            if n < 0:
                n = -1
            elif self.pages(n) > width:
                self.err |= DEVERR_PAGE
                n = self.length[s]
            want.append(n)
            if n < self.length[s]:
                for i in range(self.pages(n), self.pages(self.length[s])):
                    self._take(self.table[s, i], -1)
                    self.table[s, i] = -1
                self.length[s] = n
        free, before, at = self.free(), self.ref.copy(), 0
        for s, n in enumerate(want):
            if n <= self.length[s]:
                continue
            have, need = self.pages(self.length[s]), self.pages(n) - self.pages(self.length[s])
            used = self.length[s] % self.ps if self.length[s] > 0 else 0
            last = self.table[s, have - 1] if used else -1
            cow = bool(used) and before[last] > 1
            at += need + cow
            if at > len(free):
                self.err |= DEVERR_NO_PAGES
                continue
            taken = free[at - need - cow: at]
            first = have - cow
            self.table[s, first:first + len(taken)] = taken
            for p in taken:
                self.ref[p] = 1
            if cow:
                self.ref[last] -= 1
                for x in (self.k, self.v):
                    if x is not None:
                        x[:, taken[0], :, :used] = x[:, last, :, :used]
            self.length[s] = n

    def compact(self) -> int:
        live = [p for p in range(len(self.ref)) if self.ref[p] > 0]
        n = len(live)
        src, dst = [p for p in live if p >= n], [p for p in range(n) if self.ref[p] <= 0]
        place = dict(zip(src, dst))
        for a, b in place.items():
            self.ref[b], self.ref[a] = self.ref[a], 0
            for x in (self.k, self.v):
                if x is not None:
                    x[:, b] = x[:, a]
        for s in range(len(self.length)):
            for i in range(self.pages(self.length[s])):
                self.table[s, i] = place.get(int(self.table[s, i]), self.table[s, i])
        return n

    def write(self, layer, k_new, v_new):
        """k_new, v_new [n_seq][n_new][heads][head dim]."""
        n_new = k_new.shape[1]
        for s in range(len(self.length)):
            for i in range(n_new):
                pos = self.length[s] - n_new + i
                if self.length[s] < 0 or pos < 0:
                    continue
                p = self.table[s, pos // self.ps]
                if not 0 <= p < len(self.ref):
                    self.err |= DEVERR_PAGE
                elif self.ref[p] > 1:
                    self.err |= DEVERR_SHARED
                else:
                    self.k[layer, p, :, pos % self.ps] = k_new[s, i]
                    self.v[layer, p, :, pos % self.ps] = v_new[s, i]

    def rows(self, layer, s):
        """Keys and values of a sequence in order, fp64: [n][heads][head dim] each."""
        at = np.arange(max(0, self.length[s]))
        p = self.table[s][at // self.ps]
        return self.k[layer][p, :, at % self.ps].astype(np.float64), self.v[layer][p, :, at % self.ps].astype(np.float64)


def prefix_attention(q, cache: Cache, layer, scale, causal):
    """q [n_seq][n_q][H][D] (fp64) over each sequence's cached keys: out like q, lse [n_seq][n_q][H], and the
    same weights over |v| (for tolerances). Query i of a sequence of n tokens sees tokens j < n, or with
    `causal` j <= n - n_q + i. A query that sees nothing, or scores of -inf only: out 0, lse -inf. Sequences that
    are absent: NaN (nothing is written there)."""
    n_seq, n_q, H, D = q.shape
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse = np.full((n_seq, n_q, H), np.nan)
    for s in range(n_seq):
        n = int(cache.length[s])
        if n < 0:
            continue
        k, v = cache.rows(layer, s)
        group = H // cache.k.shape[2]
        for i in range(n_q):
            seen = max(0, n - n_q + i + 1) if causal else n
            for h in range(H):
                z = scale * (k[:seen, h // group] @ q[s, i, h])
                m = z.max() if seen else -np.inf
                if m == -np.inf:
                    out[s, i, h], mag[s, i, h], lse[s, i, h] = 0.0, 0.0, -np.inf
                    continue
                p = np.exp(z - m)
                out[s, i, h] = p @ v[:seen, h // group] / p.sum()
                mag[s, i, h] = p @ np.abs(v[:seen, h // group]) / p.sum()
                lse[s, i, h] = m + np.log(p.sum())
    return out, mag, lse
