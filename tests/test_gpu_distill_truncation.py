"""What the tensor cores' cut partial sums do to the logits of a distillation step, and what its factor takes back (GPU).

A contraction loses half of the last bit of its partial sum per 16 terms in the mean.  Hidden units in no particular order make the partial sum
grow to the logit evenly in the mean: 0.35 x 2^-23 / 2 = 2.1e-8 of the logit per step if it does so exactly, less if terms of both signs
make it wander (the sign of what is cut wanders along).  The step's factor gives 1.6e-8 back, so between -1.6e-8 and 0.5e-8 per step could
be left; that it lies within 0.6e-8 of 0 is what tells the factor from none at all (1.27e-8 and more).
"""

import math

import numpy as np
import pytest
import torch

from oracle import distill as od
from test_gpu_distill import Case, _ais, _np

pytestmark = pytest.mark.gpu

PER_STEP = 1.6e-8


def _hidden(kind, T, d, gen):
    H = torch.randn(T, d, generator=gen, device="cuda") * (1.0 + 2.0 * torch.rand(T, 1, generator=gen, device="cuda"))
    if kind == "outliers":
        H[:, torch.randperm(d, generator=gen, device="cuda")[:4]] *= 60.0
    if kind == "heavy tails":                                 # Student's t with three degrees of freedom
        H *= torch.rsqrt(sum(torch.randn(T, d, generator=gen, device="cuda") ** 2 for _ in range(3)) / 3.0 + 1e-6)
    return H.to(torch.bfloat16)


@pytest.mark.parametrize("kind", ["normal", "heavy tails", "outliers"])
@pytest.mark.parametrize("d", [1024, 4096, 5120])
def test_the_mean_shortfall_is_taken_back(kind, d):
    T, V = 2048, 1024
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    H = _hidden(kind, T, d, gen)
    W = (torch.randn(V, d, generator=gen, device="cuda") * (1.28 / math.sqrt(d))).to(torch.bfloat16)
    x = H.double() @ W.double().t()
    z, ids = x.max(dim=1)
    st = _ais().DistillStep(T, d, V, 1, want_grad=False)
    st.step(H, W, ids.int()[:, None].contiguous(), torch.zeros(T, 1, device="cuda"))
    got = st.lse.double() - st.kl.double()                    # one entry of probability 1: kl = lse - x
    slope = float(((got - z) * z).sum() / (z * z).sum())
    assert abs(slope) <= 0.6e-8 * d / 16


@pytest.mark.parametrize("d", [256, 4096])
@pytest.mark.parametrize("tau", [1.0, 0.5])
def test_contractions_without_rounding(d, tau):
    """One hidden unit per row, a power of two: every product and partial sum is a bf16 number and nothing is cut, so a logit is off by what the
    factor adds, 1.6e-8 of it per step, and its own rounding to fp32; the log-sum-exp and kl follow (1.5e-5: test_gpu_sample.py)."""
    T, V, K = 130, 1024, 16
    rng = np.random.default_rng(d)
    H = np.zeros((T, d))
    H[np.arange(T), rng.integers(0, d, T)] = 8.0
    W = rng.integers(-16, 17, (V, d)) / 8.0                   # logits in [-16, 16]
    st = _ais().DistillStep(T, d, V, K, temperature=tau)
    bf = lambda a: torch.from_numpy(a).to(torch.bfloat16).cuda()  # noqa: E731
    Hg, Wg = bf(H), bf(W)
    ids = torch.from_numpy(np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32)).cuda()
    t = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).cuda()
    st.step(Hg, Wg, ids, t)
    torch.cuda.synchronize()
    assert np.array_equal(_np(Hg), H) and np.array_equal(_np(Wg), W)
    r = od.distill(H, W, ids.cpu().numpy(), _np(t), np.ones(T), tau)
    dx = (PER_STEP * d / 16 + 2.0 ** -23) * 16.0 / tau        # (the factor is a float, too)
    assert (np.abs(_np(st.lse) - r["lse"]) <= dx + 1.5e-5 + 2.0 ** -24 * np.abs(r["lse"])).all()
    assert (np.abs(_np(st.kl) - r["kl"]) <= 2 * dx + 1.5e-5 + 2.0 ** -24 * np.abs(r["kl"])).all()


@pytest.mark.parametrize("T", [130, 2100])                    # one row tile per CTA, and two
def test_the_log_probability_pass_has_the_same_logits_without_the_factor(T):
    """H and W through the GRPO step's forward pass: the same sums of products.  A factor 1 + f moves a log-sum-exp by f sum p x, and by
    f^2 times a variance; each of the two has its own fp32 exponentials and sums (1.5e-5) and the rounding of its result."""
    d, V = 2048, 8192
    c = Case(T, d, V, 8, seed=36)
    st = c.run(c.step(grad=False))
    step = _ais().AisStep(T, d, V, 1, 1, 128)
    step.forward(c.H, c.W, torch.zeros(T, dtype=torch.int32, device="cuda"), c.mask)
    torch.cuda.synchronize()
    live = c.mask != 0
    x = (c.H.double() @ c.W.double().t())[live]
    moved = PER_STEP * d / 16 * (torch.softmax(x, dim=1) * x).sum(dim=1)
    diff = (st.lse.double() - step.lse_train[:T].double())[live] - moved
    assert (diff.abs() <= 3e-5 + 2.0 ** -23 * st.lse[live].double().abs()).all(), float(diff.abs().max())
