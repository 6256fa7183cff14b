"""The 8-bit draft cache and the attention of several rows in fp64, each from its
definition: e4m3 codes over a power-of-two scale per block, and softmax attention
over the slots that a row sees."""
from __future__ import annotations

import numpy as np

from .cache import attend
from .draft import rmsnorm

E_MIN, E_MAX = -110, 119


def e4m3_table() -> np.ndarray:
    """[256] the values of the codes: sign, 4 exponent bits (bias 7), 3 fraction
    bits; the two codes of seven ones are NaN."""
    v = np.zeros(256)
    for c in range(256):
        k, f = (c >> 3) & 15, c & 7
        x = np.nan if c & 127 == 127 else (8 + f) * 2.0 ** (k - 10) if k else f * 2.0 ** -9
        v[c] = -x if c & 128 else x
    return v


_POSITIVE = e4m3_table()[:127]


def e4m3_round(y: np.ndarray) -> np.ndarray:
    """The nearest of the values that a code can have, ties to the even code;
    larger ones than 448 are 448, what is not finite is NaN."""
    a = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    r = _POSITIVE[np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)]
    return np.where(np.isfinite(y), np.copysign(r, y), np.nan)


def scale_exponent(x: np.ndarray) -> int:
    """The exponent of the scale that the values x need."""
    fin = np.abs(x[np.isfinite(x)])
    top = float(fin.max()) if fin.size else 0.0
    e = E_MIN
    while e < E_MAX and top > 448.0 * 2.0 ** e:
        e += 1
    return e


def write_block(held: np.ndarray, e_held, rows: np.ndarray):
    """held [m, d]: values of the codes of a block's first m rows, e_held their
    scale's exponent (unused where m = 0); rows [n, d]: what is written behind
    them.  Returns the codes' values [m + n, d] and the exponent."""
    e = scale_exponent(rows)
    if len(held):
        e = max(e, e_held)
        held = e4m3_round(held * 2.0 ** (e_held - e))
    return np.concatenate([held.reshape(-1, rows.shape[1]), e4m3_round(rows * 2.0 ** -e)]), e


def rotate(x: np.ndarray, pos: int, theta: float) -> np.ndarray:
    """Pairs (x_i, x_{i + d/2}) by the angle pos * theta^(-2i/d), all in fp64."""
    h = x.shape[-1] // 2
    z = (x[..., :h] + 1j * x[..., h:]) * np.exp(1j * (float(pos) * np.power(float(theta), -np.arange(h) / h)))
    return np.concatenate([z.real, z.imag], axis=-1)


def append_row(heads: np.ndarray, nq: int, nkv: int, pos: int, theta: float, eps: float,
               q_gain=None, k_gain=None):
    """heads [nq + 2 nkv, d] of one row -> (q [nq, d], k, v [nkv, d]) before they
    are rounded."""
    q, k, v = heads[:nq], heads[nq:nq + nkv], heads[nq + nkv:]
    if q_gain is not None:
        q = rmsnorm(q, q_gain, eps)
    if k_gain is not None:
        k = rmsnorm(k, k_gain, eps)
    return rotate(q, pos, theta), rotate(k, pos, theta), v


def seen_slots(v: int, window: int, n_first: int) -> np.ndarray:
    """The slots that a row sees of those below v."""
    s = np.arange(max(v, 0))
    return s[(s >= v - window) | (s < n_first)] if window else s


def attend_row(q: np.ndarray, K: np.ndarray, V: np.ndarray, v: int, window: int, n_first: int):
    """q [g, d] over the slots of K, V [>= v, d] that it sees: out, p, lse and the slots."""
    s = seen_slots(v, window, n_first)
    return attend(q, K[s], V[s]) + (s,)
