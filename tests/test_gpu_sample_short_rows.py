"""Filters given per row on rows no longer than the list that a pass keeps, a top-k beyond the row among them (GPU)."""

import numpy as np
import pytest

from test_gpu_sample import _check, _logits, _sample, _u

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 5, 1000, 1023, 1024, 1025, 1030])
def test_top_k_at_and_beyond_the_end_of_a_row(V, dtype):
    rows = 48
    rng = np.random.default_rng(V)
    x, u = _logits(rows, V, dtype, V), _u(rows, V + 1)
    k = rng.choice([V, V + 1, 1024, 1025, 2000, 2 ** 31 - 1, 0, -5, 1], rows)
    p = rng.choice([0.3, 0.9, 1.0], rows)
    m = rng.choice([0.0, 0.05], rows)
    for how in (dict(top_k=k), dict(top_k=k, top_p=p), dict(top_k=k, min_p=m), dict(top_k=k, top_p=p, min_p=m, temperature=0.8), dict(top_p=p, min_p=m)):
        _check(x, u, *_sample(x, u, **how), **how)
