"""Long-context draft cache in fp64: appended rows, attention of one query row
over given slots, block summaries and their scores, and the choice of slots
and blocks, each from its definition."""
from __future__ import annotations

import numpy as np

from .draft import rmsnorm, rope


def append_row(heads: np.ndarray, nq: int, nkv: int, pos: int, theta: float, eps: float,
               q_gain=None, k_gain=None):
    """heads [nq + 2 nkv, d] of one row -> (q [nq, d], k, v [nkv, d])."""
    q, k, v = heads[:nq], heads[nq:nq + nkv], heads[nq + nkv:]
    if q_gain is not None:
        q = rmsnorm(q, q_gain, eps)
    if k_gain is not None:
        k = rmsnorm(k, k_gain, eps)
    return rope(q, pos, theta), rope(k, pos, theta), v


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray):
    """q [g, d] over K, V [n, d]: (out [g, d], p [g, n], lse [g])."""
    g, d = q.shape
    if K.shape[0] == 0:
        return np.zeros((g, d)), np.zeros((g, 0)), np.full(g, -np.inf)
    s = q @ K.T / np.sqrt(d)
    m = s.max(axis=1, keepdims=True)
    e = np.exp(s - m)
    S = e.sum(axis=1, keepdims=True)
    p = e / S
    return p @ V, p, (m + np.log(S))[:, 0]


def summarize(K: np.ndarray, bs: int) -> np.ndarray:
    """K [n, d] -> [ceil(n / bs), 2, d]: channelwise min and max per block."""
    n, d = K.shape
    out = np.zeros((-(-n // bs), 2, d))
    for i in range(len(out)):
        out[i, 0] = K[i * bs: (i + 1) * bs].min(axis=0)
        out[i, 1] = K[i * bs: (i + 1) * bs].max(axis=0)
    return out


def block_scores(q: np.ndarray, summary: np.ndarray) -> np.ndarray:
    """q [g, d], summary [nblk, 2, d] -> fp32 scores [nblk]."""
    best = None
    for row in q:
        s = np.where(row >= 0, row * summary[:, 1], row * summary[:, 0]).sum(axis=1).astype(np.float32)
        best = s if best is None else np.where(np.isnan(best) | np.isnan(s), np.float32("nan"),
                                               np.maximum(best, s))
    return best


def choose(values: np.ndarray, n_take: int, n_first: int, n_last: int) -> np.ndarray:
    """Indices of the n_take largest values, in index order: the first n_first
    and last n_last before all, NaN after every number, ties to the lowest."""
    n = len(values)

    def rank(i):
        forced = i < n_first or i >= n - n_last
        nan = bool(np.isnan(values[i]))
        return (not forced, nan, 0.0 if forced or nan else -float(values[i]), i)

    return np.array(sorted(sorted(range(n), key=rank)[:n_take]), dtype=np.int64)
