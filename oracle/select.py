"""Float64 definitions of drawing a token from a row of logits and of a row's top logits (test infrastructure).

Order of a row: value descending, index ascending; entries of -inf are not part of it.  Every filter keeps a prefix of that order.
"""

from __future__ import annotations

import numpy as np


def order(x: np.ndarray) -> np.ndarray:
    """Indices of the finite entries of a row in order (0 and -0 are equal)."""
    x = np.asarray(x, dtype=np.float64)
    at = np.flatnonzero(x > -np.inf)
    return at[np.lexsort((at, -(x[at] + 0.0)))]


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, lp, lp_full, n_kept, margin) of one row; (-1, 0, 0, 0, inf) where nothing can be drawn.  margin: how far the decisions
    (length of the top-p prefix, the token) were from going another way, relative to the sums that decide them."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
        return -1, 0.0, 0.0, 0, np.inf
    temperature, top_p, min_p, u = (float(np.float32(v)) for v in (temperature, top_p, min_p, u))
    if temperature == 0.0:
        temperature, top_k = 1.0, 1
    o = order(x)
    logw = (x - x.max()) / temperature
    w = np.exp(logw)
    n = len(o) if top_k <= 0 else min(top_k, len(o))
    margin = np.inf
    if top_p < 1.0:
        e = w[o[:n]]
        total = e.sum()
        before = np.concatenate(([0.0], np.cumsum(e)[:-1]))
        margin = np.min(np.abs(before[1:] - top_p * total)) / total if n > 1 else np.inf
        n = max(1, int((before < top_p * total).sum()))
    if min_p > 0.0:
        n = max(1, int((w[o[:n]] >= min_p).sum()))
    kept = np.sort(o[:n])
    cum = np.cumsum(w[kept])
    token = kept[min(int((cum <= u * cum[-1]).sum()), n - 1)]
    margin = min(margin, np.min(np.abs(cum - u * cum[-1])) / cum[-1])
    return int(token), float(logw[token] - np.log(cum[-1])), float(logw[token] - np.log(w.sum())), n, float(margin)


def top_row(x, K, temperature=1.0):
    """(ids [K], values [K], lse) of one row; ids -1 and values -inf behind the last finite entry."""
    x = np.asarray(x, dtype=np.float64)
    ids, values = np.full(K, -1, dtype=np.int64), np.full(K, -np.inf)
    if np.isnan(x).any() or (x == np.inf).any():
        return ids, values, np.nan
    o = order(x)[:K]
    ids[:len(o)], values[:len(o)] = o, x[o]
    if not len(o):
        return ids, values, -np.inf
    z = x / temperature
    return ids, values, float(z.max() + np.log(np.exp(z - z.max()).sum()))
