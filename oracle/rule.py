"""Decode attention under a score rule, and eviction by accumulated weight, in float64
(test infrastructure).

A query's score of the row at position p, the new row being at `now`:
    s = scale q.k;  s = cap tanh(s / cap);  s = s - slope (now - p)
and a row with now - p >= window and p >= prefix is not attended.  Rows that are not
attended are left out altogether, so that infinities in them have no part.
"""

import numpy as np


def attended(pos, now, window, prefix):
    pos = np.asarray(pos, dtype=np.int64)
    if window <= 0:
        return np.ones(len(pos), dtype=bool)
    return (now - pos < window) | (pos < prefix)


def rule_weights(q, K, pos, now, scale=0.0, cap=0.0, slope=0.0, window=0, prefix=0):
    """Softmax weights [n] of one query over rows K [n, d] at positions pos."""
    q, K = np.asarray(q, np.float64), np.asarray(K, np.float64)
    seen = attended(pos, now, window, prefix)
    s = (K[seen] @ q) * (scale if scale else len(q) ** -0.5)
    if cap:
        s = cap * np.tanh(s / cap)
    s = s - slope * (now - np.asarray(pos, np.float64)[seen])
    p = np.exp(s - s.max())
    out = np.zeros(len(K))
    out[seen] = p / p.sum()
    return out


def rule_attention(q, K, V, pos, now, **rule):
    """Output [d] and weights [n] of one query."""
    p = rule_weights(q, K, pos, now, **rule)
    seen = attended(pos, now, rule.get("window", 0), rule.get("prefix", 0))
    return p[seen] @ np.asarray(V, np.float64)[seen], p


def weight_drops(w, lp, recent, m):
    """Indices, ascending, of the m candidate rows of least weight: those of rows lp ..
    len(w) - recent - 1, the earliest first among equals, a NaN below any number."""
    w = np.asarray(w, np.float64)
    cand = np.arange(lp, len(w) - recent)
    x = np.where(np.isnan(w[cand]), -np.inf, w[cand])
    nan_first = ~np.isnan(w[cand])
    order = np.lexsort((cand, x, nan_first))
    return np.sort(cand[order[:m]])
