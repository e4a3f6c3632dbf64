"""CPU oracle for norms with rotary positions and the paged 8-bit cache, with numpy.

TEST INFRASTRUCTURE ONLY, as `cache_oracle`: the slow, plain statement of what the GPU library must compute, one sequence, one
head and one page at a time, with lists for whatever grows.  Everything is fp64 but the rounding to 8 bits, which is defined in
fp32 and follows that definition operation by operation.

Pins (see tests): a norm and a page by hand; a row read back is off by at most half a code; appends in any pieces give the same
pages; references are the table entries; attention over what was read back is the plain cache's.
"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

from oracle import cache_oracle as co

LEAST = np.float32(2.0 ** -100)


def norm(x: np.ndarray, weight: Optional[np.ndarray], eps: float) -> np.ndarray:
    """One row x [d]."""
    if weight is None:
        return x.astype(np.float64)
    x = x.astype(np.float64)
    return x * weight.astype(np.float64) / math.sqrt(float((x * x).sum()) / x.shape[0] + eps)


def norm_rotate(x: np.ndarray, weight: Optional[np.ndarray], eps: float, coords: Sequence[int], axis: Sequence[int],
                freq: Sequence[float], pairing: int) -> np.ndarray:
    return co.rotate(norm(x, weight, eps), coords, axis, freq, pairing)


def page_codes(rows: np.ndarray) -> Tuple[np.ndarray, np.float32]:
    """One head's rows [page, d] of a page, as they are in the storage type: codes and scale."""
    rows = rows.astype(np.float32)
    if not np.all(np.isfinite(rows)):
        return np.zeros(rows.shape, np.int8), np.float32(math.nan)
    top = np.abs(rows).max()
    if top < LEAST:
        return np.zeros(rows.shape, np.int8), np.float32(0.0)
    inv = np.float32(1.0) / top * np.float32(127.0)
    return np.clip(np.rint(rows * inv), -127, 127).astype(np.int8), top / np.float32(127.0)


class Paged:
    """Pages of a pool, and sequences that hold them.  A sequence: its pages, and its tail's rows, [Hkv, d] keys and values
    each."""

    def __init__(self, B: int, page: int, n_pages: int, max_pages: int):
        self.page, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.pool: List[Optional[Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]]] = [None] * n_pages
        self.references = [0] * n_pages
        self.pages: List[List[int]] = [[] for _ in range(B)]
        self.tails: List[List[Tuple[np.ndarray, np.ndarray]]] = [[] for _ in range(B)]

    def length(self, b: int) -> int:
        return len(self.pages[b]) * self.page + len(self.tails[b])

    def append(self, k: np.ndarray, v: np.ndarray, counts: Optional[Sequence[int]] = None) -> None:
        """k, v [B, Hkv, n, d], as the storage type has them."""
        n = k.shape[2]
        for b in range(len(self.pages)):
            for t in range(n if counts is None else min(max(counts[b], 0), n)):
                last = len(self.tails[b]) == self.page - 1
                free = [p for p in range(self.n_pages) if self.references[p] <= 0]
                if last and (not free or len(self.pages[b]) == self.max_pages):
                    break
                self.tails[b].append((k[b, :, t], v[b, :, t]))
                if last:
                    page = free[0]
                    held = [np.stack([row[i] for row in self.tails[b]], 1) for i in (0, 1)]     # [Hkv, page, d]
                    codes = [[page_codes(h) for h in x] for x in held]
                    self.pool[page] = tuple(np.stack([c[i] for c in x]) for i in (0, 1) for x in codes)
                    self.references[page] = 1
                    self.pages[b].append(page)
                    self.tails[b] = []

    def reorder(self, parent: Sequence[int]) -> "Paged":
        to = Paged(len(parent), self.page, self.n_pages, self.max_pages)
        to.pool, to.references = self.pool, list(self.references)
        for b, p in enumerate(parent):
            if 0 <= p < len(self.pages):
                to.pages[b], to.tails[b] = list(self.pages[p]), list(self.tails[p])
        for pages, sign in ((to.pages, 1), (self.pages, -1)):
            for held in pages:
                for page in held:
                    to.references[page] += sign
        return to

    def rows(self, b: int, h: int) -> Tuple[np.ndarray, np.ndarray]:
        """Keys and values of a sequence's head [length, d], in fp64."""
        out = []
        for i in (0, 1):
            parts = [self.pool[p][i][h].astype(np.float64) * float(self.pool[p][2 + i][h]) for p in self.pages[b]]
            parts += [row[i][h][None].astype(np.float64) for row in self.tails[b]]
            out.append(np.concatenate(parts) if parts else None)
        return out[0], out[1]
