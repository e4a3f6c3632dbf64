"""CPU oracle for rotary positions and the plain cache, in fp64 with numpy.

TEST INFRASTRUCTURE ONLY, as `wave_oracle`: the slow, plain statement of what the GPU library must compute, written from the
formulas, one sequence and one head at a time.  Rows are lists of vectors; nothing is vectorised beyond a row.

Pins (see tests): a turn by hand, the turn's length, its inverse and its composition; one axis against the generator's
rotary encoding of the synthetic workloads; attention over prefix and own rows against full attention over both; weights of
one step sum to the heads' share; eviction by hand.
"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

RUNS, TURNS, LADDERS = 0, 1, 2
HALVES, NEIGHBOURS = 0, 1


def pair_plan(rot_dim: int, base: float, sections: Sequence[int], order: int) -> Tuple[List[int], List[float]]:
    """Axis and frequency (radians a position) of every pair."""
    pairs = rot_dim // 2
    assert sum(sections) == pairs
    if order == TURNS:
        axis, rest = [], list(sections)
        while any(rest):
            for a in range(len(rest)):
                if rest[a] > 0:
                    rest[a] -= 1
                    axis.append(a)
    else:
        axis = sum(([a] * n for a, n in enumerate(sections)), [])
    if order == LADDERS:
        freq = sum(([base ** (-i / n) for i in range(n)] for n in sections), [])
    else:
        freq = [base ** (-i / pairs) for i in range(pairs)]
    return axis, freq


def rotate(x: np.ndarray, coords: Sequence[int], axis: Sequence[int], freq: Sequence[float], pairing: int) -> np.ndarray:
    """One row x [d] of a token at coords [n_axes]."""
    y, pairs = x.astype(np.float64).copy(), len(axis)
    for i in range(pairs):
        a, b = (i, i + pairs) if pairing == HALVES else (2 * i, 2 * i + 1)
        angle = float(coords[axis[i]]) * freq[i]
        c, s = math.cos(angle), math.sin(angle)
        y[a], y[b] = x[a] * c - x[b] * s, x[a] * s + x[b] * c
    return y


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray) -> Tuple[np.ndarray, float, np.ndarray]:
    """One head's q [d] over rows [n, d]: output, log of the normaliser, softmax weight of every row.  No rows: zero
    and -infinity."""
    if K.shape[0] == 0:
        return np.zeros(q.shape[0]), -math.inf, np.zeros(0)
    z = K @ q / math.sqrt(q.shape[0])
    top = z.max()
    e = np.exp(z - top)
    return (e / e.sum()) @ V, top + math.log(e.sum()), e / e.sum()


def cache_attention(q: np.ndarray, K: np.ndarray, V: np.ndarray, length: int, prefix_k: Optional[np.ndarray],
                    prefix_v: Optional[np.ndarray], weights: np.ndarray, decay: float
                    ) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """One unit: its G heads' queries q [G, d], own rows K, V [capacity, d] of which `length` are in use, the prefix [P, d]
    of its KV head.  Returns (out [G, d], lse [G], the own rows' new weights [length])."""
    K, V = K[:length], V[:length]
    P = 0
    if prefix_k is not None:
        P = prefix_k.shape[0]
        K, V = np.concatenate([prefix_k, K]), np.concatenate([prefix_v, V])
    out, lse = np.zeros((q.shape[0], q.shape[1])), np.zeros(q.shape[0])
    w = decay * weights[:length] if decay > 0 else np.zeros(length)
    for g in range(q.shape[0]):
        out[g], lse[g], p = attend(q[g], K, V)
        w = w + p[P:]
    return out, lse, w


def evict(positions: Sequence[int], weights: Sequence[float], length: int, tokens: int, n_keep: int, n_sink: int,
          n_local: int) -> List[int]:
    """The old row that each row of the unit holds afterwards."""
    if length <= n_keep:
        return list(range(length))

    def worth(j):
        if positions[j] < n_sink or positions[j] >= tokens - n_local:
            return math.inf, 1
        return (-math.inf, 0) if math.isnan(weights[j]) else (float(weights[j]), 1)

    def before(j):  # ascending: the best first; a kept position beats an infinite weight, any weight no number
        held = positions[j] < n_sink or positions[j] >= tokens - n_local
        w, number = worth(j)
        return (0 if held else 1, 1 - number, 0.0 if held or not number else -w, j)

    kept = set(sorted(range(length), key=before)[:n_keep])
    movers = [j for j in range(n_keep, length) if j in kept]
    rows = []
    for j in range(n_keep):
        rows.append(j if j in kept else movers.pop(0))
    assert not movers
    return rows
