"""Float64 definition of the distillation loss against a teacher's top logits and of its gradients (test infrastructure)."""

from __future__ import annotations

import numpy as np


def _lse(z):
    m = z.max(axis=1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return (m + np.log(np.exp(z - m).sum(axis=1, keepdims=True)))[:, 0]


def distill(H, W, ids, logits, mask, temperature=1.0, teacher_lse=None, weights=None):
    """H [T, d], W [V, d], ids and logits [T, K].  Returns kl [T], lse [T], loss, dH [T, d], dW [V, d] and g [T, V], the gradient
    with respect to the unscaled logits."""
    H, W, logits = (np.asarray(a, dtype=np.float64) for a in (H, W, logits))
    ids = np.asarray(ids).astype(np.int64)
    T, V = H.shape[0], W.shape[0]
    live = np.asarray(mask) != 0
    x = H @ W.T / temperature
    lse = _lse(x)
    counts = (ids >= 0) & (ids < V)
    t = np.where(counts, logits / temperature, -np.inf)
    given = counts.any(axis=1) & (t.max(axis=1) > -np.inf)
    lse_k = np.where(given, _lse(np.where(given[:, None], t, 0.0)), 0.0)
    r = np.where(given[:, None], np.exp(t - lse_k[:, None]), 0.0)
    log_mass = np.where(given, lse_k - np.asarray(teacher_lse, dtype=np.float64), 0.0) if teacher_lse is not None else np.zeros(T)
    mass = np.exp(log_mass)
    picked = np.take_along_axis(x, np.where(counts, ids, 0), axis=1)
    with np.errstate(invalid="ignore", divide="ignore"):
        terms = np.where(r > 0, r * (np.where(r > 0, t, 0.0) - lse_k[:, None] + log_mass[:, None] - picked + lse[:, None]), 0.0)
    kl = np.where(live & given, mass * terms.sum(axis=1), 0.0)
    n = live.sum()
    w = np.asarray(weights, dtype=np.float64) if weights is not None else np.full(T, 1.0 / n if n else 0.0)
    w = np.where(live & given, w, 0.0)
    p = np.exp(x - lse[:, None])
    for k in range(ids.shape[1]):
        rows = np.flatnonzero(counts[:, k])
        p[rows, ids[rows, k]] -= r[rows, k]                     # (an id given twice counts twice)
    g = p * (w * mass / temperature)[:, None]
    return dict(kl=kl, lse=np.where(live, lse, 0.0), loss=float((w * kl).sum()), dH=g @ W, dW=g.T @ H, g=g)
