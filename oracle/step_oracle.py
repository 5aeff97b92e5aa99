"""Plain numpy float64 implementation of the bounds and the choice of pages and of the norm, written from the definitions in include/parse.h.  Test
infrastructure: the product never calls it.  (The attention over shared or chosen pages is kv_oracle's.)"""
from __future__ import annotations

import numpy as np


def page_bounds(k: np.ndarray) -> np.ndarray:
    """Keys [tokens of a page][n_kv][d] -> [n_kv][2][d], least first."""
    return np.stack([k.min(0), k.max(0)], 1)


def choose(q: np.ndarray, bounds: np.ndarray, there: np.ndarray, top: int, first: int, last: int):
    """One row and kv head: q [heads of the group][d], bounds [columns][2][d], there [columns] -> (columns taken, ascending; how far, relative to the
    scores' size, the last one taken is from the first one left out)."""
    n = len(there)
    if n <= top:
        return np.flatnonzero(there), np.inf
    score = np.zeros(n)
    with np.errstate(invalid="ignore"):
        for row in q:
            score += np.maximum(row * bounds[:, 0], row * bounds[:, 1]).sum(1)
    always = [c for c in range(n) if there[c] and (c < first or c >= n - last)]
    others = [c for c in range(n) if there[c] and first <= c < n - last]
    others.sort(key=lambda c: (-np.inf if np.isnan(score[c]) else -score[c], not np.isnan(score[c]), c))
    want = top - len(always)
    gap = np.inf
    if 0 < want < len(others):
        a, b = score[others[want - 1]], score[others[want]]
        size = np.abs(q).sum(0) @ np.abs(np.nan_to_num(bounds, posinf=0, neginf=0)).max((0, 1))
        gap = (a - b) / max(size, 1e-300) if np.isfinite(a) and np.isfinite(b) else np.inf
    return np.array(sorted(always + others[:max(want, 0)]), np.int64), gap


def rmsnorm(x, residual, weight, eps):
    """x, residual [rows][d] -> (s, y)."""
    s = x + residual if residual is not None else x
    with np.errstate(invalid="ignore", divide="ignore"):
        return s, s / np.sqrt((s * s).mean(1, keepdims=True) + eps) * weight


def e4m3_values() -> np.ndarray:
    """The 127 non-negative values of the format, ascending."""
    bits = np.arange(127)
    e, m = bits >> 3, bits & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
