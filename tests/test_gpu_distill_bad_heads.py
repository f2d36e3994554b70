"""A head that holds a NaN or an infinity: every row that it makes non-finite has zeros for gradients, and so have masked rows (GPU)."""

import pytest
import torch

from test_gpu_distill import Case, _ais

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dv", [False, True])
@pytest.mark.parametrize("dw", [False, True])
@pytest.mark.parametrize("T,V", [(140, 1024), (300, 20000)])       # dH whole, and split along the vocabulary
def test_gradients_are_zero(dv, dw, T, V):
    ais = _ais()
    c = Case(T, 256, V, 8, seed=32, dv=dv, masked=0.3)
    c.W[7, 3] = float("nan")
    st = c.run(c.step(dw=dw))
    assert not st.kl.any() and not st.dH.any() and float(st.loss) == 0
    if dw:
        assert not st.dW.any()
    assert torch.isnan(st.lse[c.mask != 0]).all() and int(st.status.item()) == ais.FLAG_NONFINITE


def test_masked_rows_beside_an_infinite_weight():
    """What W holds says nothing about rows with mask 0."""
    for dw in (False, True):
        c = Case(140, 256, 1024, 8, seed=33, masked=0.3)
        c.W[7, 3] = float("inf")
        st = c.run(c.step(dw=dw))
        assert not st.dH[c.mask == 0].any() and not st.kl[c.mask == 0].any()
