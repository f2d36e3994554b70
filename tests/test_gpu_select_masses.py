"""Filters and draws among many entries of little weight (GPU), against sums in more than 64 bits.

One entry holds nearly all of the mass and a hundred thousand others decide: where top-p cuts among them, and which of them a number u draws.
The definition is summed in long double (2^-64 relative), so the distance of every decision from its border is known; the inputs keep 2e-12 of
the row's mass, where the kernels' sums are good to 1e-12: an fp64 exponential is off by 4e-14 of itself, a thread adds up 640 of them at
most (640 x 2^-53 = 7e-14) and sums are joined without further loss.
"""

import numpy as np
import pytest
import torch

from test_gpu_sample import _ais

gpu = pytest.mark.gpu

MARGIN = 2e-12
V1, V2 = 151936, 327680


def exact(x, u, T=1.0, k=0, p=1.0):
    """(token, n_kept, lp, margin): margin in units of the whole mass."""
    ld = np.longdouble
    assert np.finfo(ld).eps < 1e-18
    x = np.asarray(x, dtype=np.float64)
    w = np.exp((x.astype(ld) - ld(x.max())) / ld(np.float32(T)))
    order = np.lexsort((np.arange(len(x)), -x))
    n = len(x) if k <= 0 else min(k, len(x))
    total, margin = w[order[:n]].sum(), np.inf
    if p < 1.0:
        before = np.concatenate(([ld(0)], np.cumsum(w[order[:n]])[:-1]))
        target = ld(np.float32(p)) * total
        margin = float(np.abs(before - target).min() / total)
        n = max(1, int((before < target).sum()))
    kept = np.sort(order[:n])
    cum = np.cumsum(w[kept])
    border = ld(np.float32(u)) * cum[-1]
    margin = min(margin, float(np.abs(cum - border).min() / cum[-1]))
    token = int(kept[int((cum <= border).sum())])
    return token, n, float((ld(x[token]) - ld(x.max())) / ld(np.float32(T)) - np.log(cum[-1])), margin


def tied(V, low, seed, levels=1, step=0.0):
    """A row whose largest entry is 0, all others `low` or one of `levels` values from there down."""
    rng = np.random.default_rng(seed)
    x = low - step * rng.integers(0, levels, V)
    x[int(rng.integers(0, V))] = 0.0
    return x


def rows_of(case):
    V, low, levels, step, ps, k = case
    out = []
    for i, p in enumerate(ps):
        x = tied(V, low, 100 * i + V % 97, levels, step).astype(np.float32).astype(np.float64)
        # the largest entry has index ~V u: numbers on both sides of it, and small ones, which fall among the others
        for u in (1e-6, 0.3, 0.7):
            out.append((x, u, p, k))
    return out


CASES = [
    (V2, -22.0, 1, 0.0, (0.99995, 0.99999, 0.9999), 0),
    (V1, -24.0, 1, 0.0, (0.9999985, 0.9999971), 0),
    (V1, -18.0, 1, 0.0, (0.999, 0.9985), 0),
    (V2, -20.0, 32, 0.125, (0.9999, 0.99995), 0),
    (V1, -9.0, 64, 0.125, (0.99, 0.95, 0.3), 0),
    (V1, -21.0, 500, 0.0078125, (0.99999, 0.999993), 0),
    (V2, -22.0, 1, 0.0, (0.99996,), 200000),
]


def test_the_inputs_keep_their_distance():
    """(What the tests below rely on; nothing here runs on the device.)"""
    for case in CASES:
        for x, u, p, k in rows_of(case):
            assert exact(x, u, k=k, p=p)[3] > MARGIN, (case, u, p)


@gpu
@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("copies", [1, 60])
def test_top_p_among_entries_of_little_weight(case, copies):
    """`copies`: alone, or among others (one CTA per row instead of several)."""
    ais = _ais()
    rows = rows_of(case)
    x = torch.from_numpy(np.stack([r[0] for r in rows])).float().cuda().repeat(copies, 1)
    u = torch.tensor([r[1] for r in rows], device="cuda").repeat(copies)
    p = torch.tensor([r[2] for r in rows], device="cuda").repeat(copies)
    got = [ais.sample(x, u, top_p=p, top_k=rows[0][3])]
    if len(set(r[2] for r in rows)) == 1:
        got.append(ais.sample(x, u, top_p=rows[0][2], top_k=rows[0][3]))
    for r in got:
        for i, (xi, ui, pi, k) in enumerate(rows):
            token, n, lp, _ = exact(xi, ui, k=k, p=pi)
            assert (r.n_kept[i::len(rows)] == n).all(), (i, n, r.n_kept[i::len(rows)].tolist())
            assert (r.tokens[i::len(rows)] == token).all(), (i, token)
            assert ((r.lp[i::len(rows)].double() - lp).abs() <= 2.0 ** -24 * abs(lp) + 1e-10).all()


def _draws(k):
    """k - 1 entries at -24 in front of one at 0, and numbers that fall between 2e-12 and 5e-12 behind the sum of j of them."""
    x = np.full(5000, -60.0)
    x[:k - 1] = -24.0
    x[k - 1] = 0.0
    w = np.exp(np.longdouble(-24.0))
    total = 1 + (k - 1) * w
    us = [np.float32((j * w + side * np.longdouble(3e-12)) / total) for j in (200, 500, 900) if j < k for side in (-1, 1)]
    return x, us


def test_draws_keep_their_distance():
    for k in (600, 1000):
        x, us = _draws(k)
        assert all(exact(x, u, k=k)[3] > MARGIN for u in us)


@gpu
@pytest.mark.parametrize("k", [600, 1000])
def test_draws_from_a_list_of_entries_of_little_weight(k):
    ais = _ais()
    x, us = _draws(k)
    r = ais.sample(torch.from_numpy(x).float().cuda().repeat(len(us), 1), torch.tensor(us, device="cuda"), top_k=k)
    for i, u in enumerate(us):
        token, n, lp, _ = exact(x, u, k=k)
        assert int(r.tokens[i]) == token and int(r.n_kept[i]) == n
        assert abs(float(r.lp[i]) - lp) <= 2.0 ** -24 * abs(lp) + 1e-10
