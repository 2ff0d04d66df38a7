"""fp64 definitions of the two decode forms that attend more than, or less than, one sequence's rows -- TEST
INFRASTRUCTURE ONLY, like eigen_attention.py beside it.

* attention of drafted tokens arranged as a tree: each attends the cached rows and the drafted tokens its mask names;
* decode over a selection of blocks: the blocks with the highest upper bound on their scores.

One K/V head, stateless, ordinary three-pass softmax over the rows that take part.  Rows are the rank-r rows as the cache
holds them; queries are rank-r coordinates (to_rank_space of the query).  Pins: tests/test_oracle_tree_sparse_pins.py.
"""
from __future__ import annotations

import math
from typing import List, Sequence, Tuple

import numpy as np

from .eigen_attention import lift, softmax_rows

F64 = np.float64


def mask_bits(mask: int, T: int) -> List[int]:
    """The drafted tokens a mask names; bits from T on name nothing."""
    return [s for s in range(T) if (int(mask) >> s) & 1]


def tree_depth(mask: int, t: int, T: int) -> int:
    """How far behind the cached rows token t sits: the number of other tokens its mask names."""
    return len([s for s in mask_bits(mask, T) if s != t])


def tree_weights(qp: np.ndarray, Kp: np.ndarray, kn: np.ndarray, masks: Sequence[int], d_head: int, slope: float = 0.0):
    """Scores and softmax weights of one query head: qp [T, r], cached Kp [n, r], drafted kn [T, r].  Returns
    (rows taking part per token, weights per token): row j < n is cached row j, row n + s drafted token s."""
    T, n = len(masks), Kp.shape[0]
    depth = [tree_depth(masks[t], t, T) for t in range(T)]
    rows_of, weights = [], []
    for t in range(T):
        seen = mask_bits(masks[t], T)
        K = np.concatenate([Kp, kn[seen]], axis=0)
        s = (K @ qp[t]) / math.sqrt(d_head)
        if slope:
            pos = np.concatenate([np.arange(n, dtype=F64), [n + depth[u] for u in seen]])
            s = s - float(slope) * ((n + depth[t]) - pos)
        rows_of.append(list(range(n)) + [n + u for u in seen])
        weights.append(softmax_rows(s[None, :])[0] if K.shape[0] else np.zeros(0))
    return rows_of, weights


def tree_head(qp: np.ndarray, Kp: np.ndarray, Vp: np.ndarray, kn: np.ndarray, vn: np.ndarray, masks: Sequence[int],
              U_V: np.ndarray, lowrank_out: bool = False, slope: float = 0.0) -> np.ndarray:
    """Outputs [T, d_h] (or [T, r_V]) of one query head; a token that attends nothing gets zeros."""
    V = np.concatenate([np.asarray(Vp, F64), np.asarray(vn, F64)], axis=0)
    rows_of, weights = tree_weights(np.asarray(qp, F64), np.asarray(Kp, F64), np.asarray(kn, F64), masks, U_V.shape[0], slope)
    o = np.stack([w @ V[rows] if rows else np.zeros(V.shape[1]) for rows, w in zip(rows_of, weights)])
    return o if lowrank_out else lift(o, U_V)


def block_bounds(Kp: np.ndarray, block: int) -> Tuple[np.ndarray, np.ndarray]:
    """Per-channel minima and maxima of every complete block of rows: two arrays [n // block, r]."""
    whole = Kp.shape[0] // block
    x = np.asarray(Kp)[:whole * block].reshape(whole, block, Kp.shape[1])
    return x.min(axis=1), x.max(axis=1)


def block_score(qp: np.ndarray, lo: np.ndarray, hi: np.ndarray, d_head: int) -> float:
    """An upper bound on the scores of the query qp [r] against any row between lo and hi."""
    return float(sum(max(q * a, q * b) for q, a, b in zip(qp, lo, hi))) / math.sqrt(d_head)


def choose_blocks(qps: np.ndarray, Kp: np.ndarray, block: int, n_blocks: int, sink: int, recent: int, d_head: int,
                  slope: float = 0.0) -> List[int]:
    """Blocks that the query heads qps [g, r] of one K/V head attend over its n rows, ascending."""
    n = Kp.shape[0]
    have = -(-n // block)
    if have <= n_blocks:
        return list(range(have))
    lo, hi = block_bounds(Kp, block)
    middle = list(range(sink, have - recent))
    score = {}
    for j in middle:
        s = max(block_score(q, lo[j], hi[j], d_head) for q in qps)
        score[j] = s - float(slope) * ((n - 1) - ((j + 1) * block - 1)) if slope else s
    best = sorted(middle, key=lambda j: (-score[j], j))[:n_blocks - sink - recent]
    return sorted(list(range(sink)) + best + list(range(have - recent, have)))


def blocks_head(qp: np.ndarray, Kp: np.ndarray, Vp: np.ndarray, blocks: Sequence[int], block: int, U_V: np.ndarray,
                lowrank_out: bool = False, slope: float = 0.0) -> np.ndarray:
    """Decode of one query [r] over the rows of the given blocks: [d_h] (or [r_V])."""
    Kp, Vp = np.asarray(Kp, F64), np.asarray(Vp, F64)
    n = Kp.shape[0]
    rows = [j for b in blocks for j in range(b * block, min(n, (b + 1) * block))]
    s = (Kp[rows] @ qp) / math.sqrt(U_V.shape[0])
    if slope:
        s = s - float(slope) * ((n - 1) - np.asarray(rows, dtype=F64))
    o = softmax_rows(s[None, :])[0] @ Vp[rows]
    return o if lowrank_out else lift(o, U_V)
