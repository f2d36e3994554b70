"""Hand-checked values and differences that pin the float64 definitions of sampling, top logits and distillation (CPU)."""

import numpy as np
import pytest

from oracle import distill as od
from oracle import select as osel

L = np.log


def test_prefix_filters_on_a_row_of_known_probabilities():
    p = np.array([0.1, 0.4, 0.2, 0.2, 0.1])
    x = L(p)
    assert list(osel.order(x)) == [1, 2, 3, 0, 4]                             # equal values in the order of their indices
    assert osel.sample_row(x, 0.0)[0] == 0 and osel.sample_row(x, 0.45)[0] == 1 and osel.sample_row(x, 0.99)[0] == 4
    t, lp, full, n, _ = osel.sample_row(x, 0.0, top_k=2)                     # keeps 1 and 2
    assert (t, n) == (1, 2) and lp == pytest.approx(L(0.4 / 0.6)) and full == pytest.approx(L(0.4))
    assert osel.sample_row(x, 0.7, top_k=2)[0] == 2
    assert osel.sample_row(x, 0.5, top_p=0.39)[3] == 1 and osel.sample_row(x, 0.5, top_p=0.41)[3] == 2
    assert osel.sample_row(x, 0.5, top_k=3, top_p=0.49)[3] == 1 and osel.sample_row(x, 0.5, top_k=3, top_p=0.51)[3] == 2   # 0.4 of 0.8
    assert osel.sample_row(x, 0.5, min_p=0.49)[3] == 3 and osel.sample_row(x, 0.5, min_p=1.0)[3] == 1
    assert osel.sample_row(x, 0.5, top_p=0.0)[3] == 1
    assert osel.sample_row(x, 0.9, temperature=0.0)[:2] == (1, 0.0)
    assert osel.sample_row(x, 0.5, temperature=0.5)[2] == pytest.approx(L(0.16 / 0.26))
    assert osel.sample_row([-np.inf, 1.0], 0.0)[0] == 1 and osel.sample_row([-np.inf] * 2, 0.5)[0] == -1
    assert osel.sample_row([0.0, np.nan], 0.5)[0] == -1


def test_top_row_pads_and_orders_ties():
    ids, v, lse = osel.top_row([1.0, -np.inf, 2.0, 1.0], 4)
    assert list(ids) == [2, 0, 3, -1] and v[3] == -np.inf and lse == pytest.approx(L(np.exp(2) + 2 * np.exp(1)))


def test_distillation_of_one_row_by_hand():
    # one hidden unit, three logits 0, ln 2, ln 5 -> p = 1/8, 2/8, 5/8; teacher 1/4 and 3/4 on entries 0 and 2
    H, W = np.array([[1.0]]), np.array([[0.0], [L(2)], [L(5)]])
    r = od.distill(H, W, [[2, 0]], [[L(3), 0.0]], [1])
    assert r["kl"][0] == pytest.approx(0.25 * L(0.25 / 0.125) + 0.75 * L(0.75 / 0.625))
    assert np.allclose(r["g"][0], [1 / 8 - 1 / 4, 2 / 8, 5 / 8 - 3 / 4])
    # the teacher's own probabilities 0.15 and 0.45: mass 0.6
    r = od.distill(H, W, [[2, 0]], [[L(3), 0.0]], [1], teacher_lse=[L(4 / 0.6)])
    assert r["kl"][0] == pytest.approx(0.15 * L(0.15 / 0.125) + 0.45 * L(0.45 / 0.625))
    assert np.allclose(r["g"][0], 0.6 * np.array([1 / 8 - 1 / 4, 2 / 8, 5 / 8 - 3 / 4]))
    # padding, an entry of no probability, an id given twice, a masked row
    r = od.distill(np.ones((2, 1)), W, [[-1, 2, 2, 0], [2, 0, 1, -1]], [[9.0, 0.0, 0.0, -np.inf], [0.0] * 4], [1, 0])
    assert r["kl"][0] == pytest.approx(0.5 * (L(0.5 / 0.625) * 2)) and r["kl"][1] == 0
    assert np.allclose(r["g"][0], [1 / 8, 2 / 8, 5 / 8 - 1]) and not r["g"][1].any()


@pytest.mark.parametrize("full", [False, True])
def test_gradients_against_differences(full):
    rng = np.random.default_rng(3)
    H, W = rng.normal(size=(3, 4)), rng.normal(size=(11, 4))
    ids = np.stack([rng.permutation(11)[:5] for _ in range(3)])
    ids[1, 3] = ids[1, 0]
    ids[2, 4] = -1
    args = dict(temperature=1.7, teacher_lse=rng.normal(size=3) + 3.0 if full else None, weights=np.array([0.5, -2.0, 1.0]))
    t, mask = rng.normal(size=(3, 5)), np.ones(3)
    r = od.distill(H, W, ids, t, mask, **args)
    h = 1e-6
    for name, a in (("dH", H), ("dW", W)):
        num = np.zeros_like(a)
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            up = od.distill(H, W, ids, t, mask, **args)["loss"]
            a[i] = keep - h
            num[i] = (up - od.distill(H, W, ids, t, mask, **args)["loss"]) / (2 * h)
            a[i] = keep
        # the truncation error of a central difference is h^2 times a third derivative of order one, its rounding 1e-16 / h
        assert np.abs(num - r[name]).max() <= 1e-8
