"""Rows whose first entries are banned, and rows of low logits, against the float64 definitions (GPU).

The log-sum-exp of a row is a sum about a reference that the row itself has to give: a reference of 0 for logits near -87 leaves a sum of
numbers below 2^-126, which the exponential flushes.  Tolerances as in test_gpu_sample.py: 2^-24 of the value and 1.5e-5.
"""

import numpy as np
import pytest
import torch

from test_gpu_sample import DTYPES, _ais, _check, _check_top, _sample, _u

pytestmark = pytest.mark.gpu


def _rows(rows, V, dtype, mean, sd, seed, keep, lead=0, ld=None):
    """[rows, V] of normal logits with -inf outside keep(indices), in a buffer that starts `lead` elements late."""
    rng = np.random.default_rng(seed)
    x = mean + sd * rng.standard_normal((rows, V))
    x[:, ~keep(np.arange(V))] = -np.inf
    ld = ld or V
    buf = torch.full((lead + rows * ld + 16,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = buf[lead:lead + rows * ld].view(rows, ld)[:, :V]
    view.copy_(torch.from_numpy(x))
    return view


def _check_all(x, K, T, pick):
    """Log-sum-exps, ids and values of the rows in `pick`, and tokens, counts and both log-probs, with top-k and greedy."""
    u = _u(x.shape[0], 3)
    sub = torch.tensor(pick, device="cuda")
    r = _ais().top_logits(x, K, temperature=T)
    _check_top(x[sub], K, T, _ais().TopLogits(*(t[sub] for t in r)))
    for how in (dict(top_k=K, temperature=T), dict(temperature=0.0)):
        r, status = _sample(x, u, **how)
        _check(x[sub], u[sub], _ais().Sampled(*(t[sub] for t in r)), status, **how)


# a row of a batch of 150 or more belongs to one CTA, one row to eight
@pytest.mark.parametrize("rows,pick", [(1, [0]), (3, [0, 1, 2]), (150, [0, 77, 149])])
@pytest.mark.parametrize("mean,sd,T", [(-86.0, 2.0, 1.0), (-88.0, 2.0, 1.0), (-90.0, 2.0, 1.0), (-100.0, 1.0, 1.0), (-17.6, 0.5, 0.2), (-8.8, 0.1, 0.1)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_banned_prefix(rows, pick, mean, sd, T, dtype):
    V = 50000
    for banned in (8192, 16384, 20001, 40000):
        _check_all(_rows(rows, V, dtype, mean, sd, 1, lambda i: i >= banned), 20, T, pick)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mean", [-86.0, -90.0, -717.0, -735.0])
def test_a_small_allowed_set(dtype, mean):
    """What constrained decoding leaves of a row: a few entries, at the front, in the middle or at the end, or one slice of eight."""
    V = 151936
    for keep in (lambda i: i < 5, lambda i: (i >= 70000) & (i < 70040), lambda i: i >= V - 3, lambda i: i % 9973 == 0, lambda i: i >= V // 2):
        for rows in (1, 160):
            _check_all(_rows(rows, V, dtype, mean, 2.0, 2, keep), 3, 1.0, [0, rows - 1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 5, 7, 15, 31, 8200])
def test_the_ends_of_a_row_alone(dtype, V):
    """Rows of fewer entries than a 16-byte load, and rows of which nothing outside their first and last loads is left."""
    for lead in (0, 1, 3):
        for mean in (-86.0, -88.0, -95.0):
            keep = (lambda i: i >= 0) if V < 32 else (lambda i: (i < 3) | (i >= V - 3))
            _check_all(_rows(2, V, dtype, mean, 2.0, V, keep, lead=lead, ld=V + 1), min(V, 4), 1.0, [0, 1])


def test_a_bad_entry_in_front_of_the_first_finite_one():
    """NaN and +inf among banned entries are seen, whichever part of the row they stand in."""
    ais = _ais()
    V = 60000
    for rows in (1, 150):
        for at in (0, 3, 8191, 9000, 25000, 59999):
            for bad in (float("nan"), float("inf")):
                x = _rows(rows, V, "fp32", -5.0, 2.0, 4, lambda i: i >= 30000, lead=1)
                x[0, at] = bad
                status = torch.zeros(1, dtype=torch.int32, device="cuda")
                r = ais.top_logits(x, 8, status=status)
                s = ais.sample(x, _u(rows, 5), top_k=8, status=status)
                assert torch.isnan(r.lse[0]) and int(r.ids[0, 0]) == -1 and int(s.tokens[0]) == -1
                assert int(status.item()) == ais.FLAG_NONFINITE
