"""Row weights so small that a row's factor leaves the range of fp32 while its gradient does not (GPU).

The scratch of a step with dH alone holds e^x, and the dH pass multiplies the row by w M e^-lse / tau: at a log-sum-exp of 50 a weight of
1e-22 makes that 2e-44, a number of four bits, though dH itself, of the order of 1e-22, has all of bf16's.  Tolerances: test_gpu_distill.py.
"""

import pytest
import torch

from test_gpu_distill import Case, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dv", [False, True])
@pytest.mark.parametrize("dw", [False, True])
def test_small_weights_beside_large_log_sum_exps(dv, dw):
    c = Case(300, 256, 1024, 12, seed=34, dv=dv, weights=True, gain=1.0)
    c.W[:, 0] = 6.25
    c.H[:, 0] = 8.0                                           # (every logit of a row 50 higher)
    c.H[::3, 0] = 0.0
    scale = torch.ones(300, device="cuda")
    scale[:128] = 1e-22                                       # a whole row tile
    scale[140::7] = 1e-25
    scale[141::7] = 1e-27
    c.weights *= scale
    r = c.check(c.run(c.step(dw=dw)))
    assert r["lse"].max() > 50


def test_a_factor_of_one():
    """Rows whose factor happens to be 1: the two forms of the scratch are the same there."""
    c = Case(200, 256, 1024, 12, seed=35, gain=1.0)
    for _ in range(2):
        st = c.run(c.step())
        c.weights = torch.exp(st.lse)                         # w e^-lse = 1 to within its rounding, and exactly in some rows
    c.check(st)
    assert _np(st.lse).min() > 0
