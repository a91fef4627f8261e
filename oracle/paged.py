"""The paged full-context cache from its definition (include/kvr.h, kvr_paged_*):
plans in whole numbers, the bounds of full pages, and attention over all or some
of the pages in 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


class Plan:
    """Lengths, tables and the stack of free pages."""

    def __init__(self, n_seq, n_pages, page_rows, table_pages):
        self.P, self.most = page_rows, table_pages
        self.len = [0] * n_seq
        self.table = [[] for _ in range(n_seq)]
        self.stack = list(range(n_pages - 1, -1, -1))  # the last one goes first

    def plan(self, lens, n_new=0):
        """The slots [S][n_new], and which error word's bit a refusal sets (None,
        "length" or "capacity")."""
        S, P = len(self.len), self.P
        slots = np.full((S, n_new), -1, np.int32)
        for old, n in zip(self.len, lens):
            if n < 0 or n > self.most * P or n - old > n_new:
                return slots, "length"
        need = [-(-n // P) for n in lens]
        back = [t[k:] for t, k in zip(self.table, need)]
        short = sum(max(k - len(t), 0) for t, k in zip(self.table, need))
        if short > len(self.stack) + sum(map(len, back)):
            return slots, "capacity"
        for page in reversed([p for b in back for p in b]):
            self.stack.append(page)
        for s in range(S):
            del self.table[s][need[s]:]
            while len(self.table[s]) < need[s]:
                self.table[s].append(self.stack.pop())
            for t in range(lens[s] - self.len[s]):
                pos = self.len[s] + t
                slots[s, t] = self.table[s][pos // P] * P + pos % P
            self.len[s] = lens[s]
        return slots, None

    def table_array(self):
        a = np.full((len(self.table), self.most), -1, np.int32)
        for s, t in enumerate(self.table):
            a[s, :len(t)] = t
        return a


def bounds(k):
    """Least and greatest of a full page's keys [P][d], NaN where one is."""
    return np.stack((k.min(0), k.max(0)))


def score(q, least, greatest):
    """Of a page, for the query heads q [G][d] that share its KV head."""
    q, lo, hi = (np.asarray(x, np.float64) for x in (q, least, greatest))
    with np.errstate(all="ignore"):
        return (q * np.where(q > 0, hi, lo)).sum(-1).max()


def choose(q, k, page_rows, budget, window):
    """The pages of rows k [n][d] that stay for q [G][d], ascending."""
    n = len(k)
    have = -(-n // page_rows)
    if have <= budget + window:
        return list(range(have))
    old = have - window
    s = [score(q, *bounds(k[i * page_rows:(i + 1) * page_rows]))
         for i in range(old)]
    order = sorted(range(old), key=lambda i: (
        not np.isnan(s[i]), 0.0 if np.isnan(s[i]) else -s[i], i))
    return sorted(order[:budget]) + list(range(old, have))


def attend(q, k, v, scale=None):
    """One unit in 64 bits: q [G][d], k and v [n][d].  Returns out [G][d], per
    output the probability-weighted mean of |v|, and per head the greatest sum of
    |q c k c| (times the scale) of a row."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    scale = 1.0 / np.sqrt(q.shape[-1]) if scale is None else scale
    if len(k) == 0:
        return np.zeros(q.shape), np.zeros(q.shape), np.zeros(len(q))
    x = q @ k.T * scale
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, p @ np.abs(v), (np.abs(q) @ np.abs(k).T).max(-1) * scale


def rows_of(pages, n, page_rows):
    """Rows of the pages at these positions, of a sequence of n."""
    r = (np.asarray(pages, np.int64)[:, None] * page_rows
         + np.arange(page_rows)).ravel()
    return r[r < n]
