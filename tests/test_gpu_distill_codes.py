"""Distillation with dW where most logits lie far below the row's log-sum-exp (GPU).

With dW the forward pass leaves 16-bit codes of the logits, which begin at -42.  Rows of a low log-sum-exp have entries below that which
still count, so they may not stay in that form.  Tolerances: test_gpu_distill.py, which bounds every entry of dW relative to the terms that
it sums.
"""

import numpy as np
import pytest
import torch

from test_gpu_distill import Case

pytestmark = pytest.mark.gpu


def _case(h, dv, **kw):
    """Eight logits near -2.1 h[t] and the others near -4.3 h[t]."""
    c = Case(len(h), 256, 1024, 12, seed=31, dv=dv, gain=1.0, **kw)
    c.W[:, 0] = -4.3125
    c.W[:8, 0] = -2.09375
    c.H[:, 0] = torch.from_numpy(np.asarray(h))
    return c


@pytest.mark.parametrize("dv", [False, True])
@pytest.mark.parametrize("grad", [False, True])
def test_entries_far_below_a_low_log_sum_exp(dv, grad):
    c = _case(np.full(130, 10.0), dv)
    r = c.check(c.run(c.step(grad=grad, dw=True)))
    assert (r["lse"] > -20).all() and (r["lse"] < -15).all() and (np.abs(r["dW"][8:]).max(axis=1) > 0).all()


@pytest.mark.parametrize("dv", [False, True])
def test_log_sum_exps_on_both_sides_of_the_range_of_the_codes(dv):
    c = _case(np.linspace(1.0, 11.0, 300), dv, masked=0.2, weights=True)
    r = c.check(c.run(c.step(dw=True)))
    assert r["lse"].min() < -18 and r["lse"].max() > 0
