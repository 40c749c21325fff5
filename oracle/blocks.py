"""Which rows a block-sparse decode step attends to, in exact arithmetic (test
infrastructure).

Of a head of n cached rows before the step's append, blocks of 32 rows that end at or
below row n - recent are candidates.  A block is scored from the bounds of its keys
in 8 bits (see ``scores``), and where there are more than n_blocks candidates the
n_blocks of highest score are attended, the lowest index first among equals, with
every row past the candidates and the new one.
"""

import numpy as np

from .quant import BF16_MAX

BLOCK = 32


def _finite(x):
    x = np.asarray(x, dtype=np.float64)
    return np.clip(np.where(np.isnan(x), 0.0, x), -BF16_MAX, BF16_MAX)


def unit(amax):
    """t with amax / 2^t in (63.5, 127], within [-60, 50] (-60 for zero)."""
    f, e = np.frexp(np.asarray(amax, dtype=np.float64))
    t = np.where(2 * f <= 127 / 64, e - 7, e - 6)
    return np.clip(np.where(amax == 0, -60, t), -60, 50)


def scores(q, keys):
    """[blocks] scores of whole blocks of ``keys`` [32 * blocks, d] against q [G, d]:
    max over the queries of 2^(t+u) sum_c max(Q_c H_c, Q_c L_c)."""
    k = _finite(keys)
    k = k.reshape(-1, BLOCK, k.shape[-1])
    hi, lo = k.max(1), k.min(1)
    t = unit(np.maximum(np.abs(hi), np.abs(lo)).max(1))[:, None]
    hi = np.clip(np.ceil(hi / 2.0 ** t), -127, 127)
    lo = np.clip(np.floor(lo / 2.0 ** t), -127, 127)
    q = _finite(q)
    u = unit(np.abs(q).max(1))[:, None]
    qi = np.clip(np.rint(q / 2.0 ** u), -127, 127)
    dot = np.maximum(qi[:, None] * hi, qi[:, None] * lo).sum(-1)      # [G, blocks]
    return (dot * 2.0 ** (u + t.T)).max(0)


def candidates(n, recent):
    return max(0, n - recent) // BLOCK


def chosen(q, keys, n, n_blocks, recent):
    """Chosen blocks, ascending, or None where every candidate is attended."""
    cand = candidates(n, recent)
    if cand <= n_blocks:
        return None
    s = scores(q, keys[:cand * BLOCK])
    order = sorted(range(cand), key=lambda b: (-s[b], b))
    return np.array(sorted(order[:n_blocks]), dtype=np.int64)


def attended(q, keys, n, n_blocks, recent):
    """Ascending indices of the attended rows among rows 0 .. n (n: the new one)."""
    pick = chosen(q, keys, n, n_blocks, recent)
    if pick is None:
        return np.arange(n + 1)
    head = (pick[:, None] * BLOCK + np.arange(BLOCK)).reshape(-1)
    return np.concatenate([head, np.arange(candidates(n, recent) * BLOCK, n + 1)])
