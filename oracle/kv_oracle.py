"""Plain numpy float64 implementation of the paged key-value cache and of the attention over it, written from the definitions in
include/parse.h.  Test infrastructure: the product never calls it."""
from __future__ import annotations

import numpy as np


# ---- layout --------------------------------------------------------------------------------------------------------
def k_to_pages(k: np.ndarray) -> np.ndarray:
    """[tokens of a page][n_kv][d] -> [n_kv][page/16][d/8][16][8]."""
    page, n_kv, d = k.shape
    return k.transpose(1, 0, 2).reshape(n_kv, page // 16, 16, d // 8, 8).transpose(0, 1, 3, 2, 4)


def v_to_pages(v: np.ndarray) -> np.ndarray:
    """[tokens of a page][n_kv][d] -> [n_kv][page/8][d][8]."""
    page, n_kv, d = v.shape
    return v.transpose(1, 0, 2).reshape(n_kv, page // 8, 8, d).transpose(0, 1, 3, 2)


def k_from_pages(K: np.ndarray) -> np.ndarray:
    """[...][n_kv][page/16][d/8][16][8] -> [...][page][n_kv][d]."""
    n_kv, b, d8 = K.shape[-5:-2]
    x = np.moveaxis(K, -3, -2).reshape(*K.shape[:-4], b * 16, d8 * 8)
    return np.moveaxis(x, -3, -2)


def v_from_pages(V: np.ndarray) -> np.ndarray:
    """[...][n_kv][page/8][d][8] -> [...][page][n_kv][d]."""
    n_kv, b, d = V.shape[-4:-1]
    x = np.moveaxis(V, -1, -2).reshape(*V.shape[:-3], b * 8, d)
    return np.moveaxis(x, -3, -2)


# ---- bookkeeping, one sequence after another ---------------------------------------------------------------------------
class Pages:
    """Table, lengths and uses of the pages; every call returns the copies (from, to) that it asks for, in order."""

    def __init__(self, n_seqs, max_pages, n_pages, page):
        self.table = np.full((n_seqs, max_pages), -1, np.int64)
        self.len = np.zeros(n_seqs, np.int64)
        self.refs = np.zeros(n_pages, np.int64)
        self.page = page

    def free_words(self) -> np.ndarray:
        n = len(self.refs)
        bits = np.zeros(-(-n // 32) * 32, np.uint32)
        bits[:n] = self.refs == 0
        return (bits.reshape(-1, 32) << np.arange(32, dtype=np.uint32)).sum(1, dtype=np.uint32)

    def _give(self, s, c):
        if self.table[s, c] >= 0:
            self.refs[self.table[s, c]] -= 1
            self.table[s, c] = -1

    def fork(self, src, dst):
        rows, lens = self.table[src].copy(), self.len[src].copy()
        for r in rows:
            for p in r[r >= 0]:
                self.refs[p] += 1
        for d, r, n in zip(dst, rows, lens):
            for c in range(self.table.shape[1]):
                self._give(d, c)
            self.table[d], self.len[d] = r, n

    def reserve(self, n_new):
        copies, served, short = [], np.zeros(len(self.len), np.int32), False
        for s, more in enumerate(n_new):
            more, n = int(more), int(self.len[s])
            if more <= 0 or n + more > self.table.shape[1] * self.page or short:
                continue
            first = n // self.page
            begun = n % self.page != 0
            old = int(self.table[s, first]) if begun else -1
            new = list(range(-(-n // self.page), -(-(n + more) // self.page)))
            if begun and (old < 0 or self.refs[old] > 1):
                new = [first] + new
            free = np.flatnonzero(self.refs == 0)
            if len(new) > len(free):
                short = True
                continue
            for c, p in zip(new, free):
                if c == first and begun and old >= 0:
                    copies.append((old, int(p)))
                    self.refs[old] -= 1
                self.table[s, c] = p
                self.refs[p] = 1
            self.len[s] = n + more
            served[s] = 1
        return copies, served

    def trim(self, keep=None, window=0, sinks=0):
        for s in range(len(self.len)):
            if keep is not None:
                self.len[s] = min(self.len[s], max(int(keep[s]), 0))
            n = self.len[s]
            for c in range(self.table.shape[1]):
                a, b = c * self.page, (c + 1) * self.page
                if a >= n or (window > 0 and a >= sinks and b <= n - window + 1):
                    self._give(s, c)

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] == 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        for p, h in zip(movers, holes):
            self.table[self.table == p] = h
            self.refs[h], self.refs[p] = self.refs[p], 0
        return list(zip(movers, holes)), live


# ---- values ----------------------------------------------------------------------------------------------------------
def rotate(x: np.ndarray, rope: np.ndarray) -> np.ndarray:
    """x [rows][heads][d], rope [rows][d] (cosines, sines of each row's position)."""
    h = x.shape[2] // 2
    c, s = rope[:, None, :h], rope[:, None, h:]
    return np.concatenate([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], 2)


def visible(i: int, there: np.ndarray, window: int, sinks: int) -> np.ndarray:
    """Which positions j (there[j]: its page is there) the row at position i sees."""
    j = np.arange(len(there))
    seen = (j <= i) & there
    return seen & ((j > i - window) | (j < sinks)) if window > 0 else seen


def attend_row(q, k, v, seen, scale):
    """q [heads][d], k, v [tokens][n_kv][d] -> (o, lse, the same mean of |v|, largest scale * |q| . |k|) per head."""
    heads, n_kv = q.shape[0], k.shape[1]
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, big = np.full(heads, -np.inf), np.zeros(heads)
    idx = np.flatnonzero(seen)
    if len(idx):
        for h in range(heads):
            kh, vh = k[idx, h // (heads // n_kv)], v[idx, h // (heads // n_kv)]
            s = scale * (kh @ q[h])
            m = s.max()
            p = np.exp(s - m)
            o[h], mag[h] = p @ vh / p.sum(), p @ np.abs(vh) / p.sum()
            lse[h] = m + np.log(p.sum())
            big[h] = abs(scale) * (np.abs(kh) @ np.abs(q[h])).max()
    return o, lse, mag, big
