"""Distillation at sizes whose passes take two row tiles per CTA and pace their CTAs (GPU).

The reference is the definition in 64 bits, on the device.  Elementwise tolerances are those of test_gpu_distill.py.  By norm: a gradient
entry is rounded to bf16 in the scratch and once more in the result, each off by a number between -2^-8 and 2^-8 of its size, at most 2^-8 /
sqrt(3) rms, and with dW by the codes' 8e-4 at most; in a sum over rows (columns) whose other factor is random these errors add up as their
squares do, like the sum itself: sqrt(2 / 3 x 2^-16 + 8e-4^2) = 3.3e-3 of it; 4e-3 is allowed.  A row tile has few rows, of which one may outweigh the others, so each of
the roundings is taken at its largest there: 2 x 2^-8 + 8e-4 = 8.6e-3.  The norm of dW is taken apart over the
vocabulary entries that no teacher lists as well: nothing but p is in them.
"""

import numpy as np
import pytest
import torch

from test_gpu_distill import STEP16, _ais

pytestmark = pytest.mark.gpu

NORM, TILE_NORM = 4e-3, 8.6e-3


class Big:
    def __init__(self, T, d, V, K, seed, tau=1.0, full=False, weights=False, dv=False, pad=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        self.tau, self.dv, self.ldh = tau, dv, d + pad
        buf = torch.full((T, d + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.H = buf[:, :d]
        self.H.copy_(rnd(T, d) * (1.0 + 2.0 * torch.rand(T, 1, generator=gen, device="cuda")))
        self.W = (rnd(V, d) * (1.28 / np.sqrt(d))).to(torch.bfloat16)
        z = (self.H @ self.W.t()).float() + rnd(T, V)
        z[:, ::7] = -1e30                                     # (columns that no teacher lists)
        self.logits, ids = z.topk(K, dim=1)
        self.ids = ids.to(torch.int32)
        self.lse = torch.logsumexp(z / tau, dim=1) + 0.1 if full else None
        self.weights = rnd(T) if weights else None
        self.mask = (torch.rand(T, generator=gen, device="cuda") < 0.9).to(torch.uint8)
        self.mask[0] = 1

    def step(self, grad=True, dw=False, fill=True, **kw):
        T, d = self.H.shape
        st = _ais().DistillStep(T, d, self.W.shape[0], self.ids.shape[1], temperature=self.tau, want_grad=grad, want_dw=dw, ldh=self.ldh,
                                w_layout=_ais().W_DV if self.dv else _ais().W_VD, **kw)
        if fill:
            st.workspace.fill_(255)
        return st

    def run(self, st):
        st.step(self.H, self.W.t().contiguous() if self.dv else self.W, self.ids, self.logits, teacher_lse=self.lse, mask=self.mask, weights=self.weights)
        torch.cuda.synchronize()
        return st

    def check(self, st, flags=0):
        live = self.mask != 0
        H, W = torch.nan_to_num(self.H).double(), self.W.double()
        T, d = H.shape
        V = W.shape[0]
        x = H @ W.t() / self.tau
        dx = (d / 16) * 2.0 ** -23 * (H.abs() @ W.abs().t()).amax(dim=1) / self.tau
        lse = torch.logsumexp(x, dim=1)
        t, ids = self.logits.double() / self.tau, self.ids.long()
        log_q = t - (torch.logsumexp(t, dim=1) if self.lse is None else self.lse.double())[:, None]
        q = log_q.exp()
        mass = q.sum(dim=1)
        kl = torch.where(live, (q * (log_q - x.gather(1, ids) + lse[:, None])).sum(dim=1), 0.0)
        w = torch.where(live, self.weights.double() if self.weights is not None else 1.0 / live.sum(), 0.0)
        tol = mass * (2 * dx + 1.5e-5) + 2.0 ** -24 * kl.abs()
        assert ((st.kl - kl).abs() <= tol).all()
        assert ((st.lse - torch.where(live, lse, 0.0)).abs() <= dx + 1.5e-5 + 2.0 ** -24 * lse.abs()).all()
        assert abs(float(st.loss) - float((w * kl).sum())) <= float((w.abs() * tol).sum()) + 2.0 ** -23 * abs(float((w * kl).sum()))
        assert int(st.status.item()) == flags
        if st.dH is None and st.dW is None:
            return
        p = (x - lse[:, None]).exp_()
        del x
        row = (w * mass / self.tau).abs()[:, None]
        g = p * mass[:, None]
        g.scatter_add_(1, ids, -q)
        g *= (w / self.tau)[:, None]
        dg = STEP16 * g.abs() + p * row * (2 * dx + 2e-5 + (8e-4 if st.dW is not None else 0.0))[:, None]
        if st.dH is not None:
            dH = g @ W
            tol = dg @ W.abs() + (V / 16 + 1) * 2.0 ** -23 * (g.abs() @ W.abs()) + 2.0 ** -23 * (p @ W.abs()) * row
            tol += STEP16 * (dH.abs() + tol) + 1e-38
            assert ((st.dH - dH).abs() <= tol).all()
            assert not st.dH[~live].any()
            assert (st.dH - dH).norm() <= NORM * dH.norm()
            for tile in range(0, T, 128):                     # (and of every row tile by itself)
                assert (st.dH[tile:tile + 128] - dH[tile:tile + 128]).norm() <= TILE_NORM * dH[tile:tile + 128].norm()
        if st.dW is not None:
            dW = g.t() @ H
            tol = dg.t() @ H.abs() + (T / 16 + 1) * 2.0 ** -23 * (g.abs().t() @ H.abs())
            tol += STEP16 * (dW.abs() + tol) + 1e-38
            got = (st.dW.t() if self.dv else st.dW).double()
            assert ((got - dW).abs() <= tol).all()
            listed = torch.zeros(V, dtype=torch.bool, device="cuda")
            listed[ids[live].flatten()] = True
            assert (~listed).sum() > V // 10
            for part in (listed, ~listed):
                assert (got[part] - dW[part]).norm() <= NORM * dW[part].norm()


WHAT = [(False, False), (True, False), (False, True), (True, True)]


@pytest.mark.parametrize("dv", [False, True])
@pytest.mark.parametrize("grad,dw", WHAT)
@pytest.mark.parametrize("T,d,V,K", [(2100, 2048, 32008, 17),      # 17 row tiles: the last pair has one
                                     (2305, 1024, 65536, 64)])
def test_pairs_of_row_tiles(T, d, V, K, grad, dw, dv):
    c = Big(T, d, V, K, seed=T, dv=dv, pad=16, full=dw)
    c.mask[128:256] = 0                                       # the second tile of a pair
    c.mask[512:640] = 0                                       # the first of one
    c.mask[1024:1280] = 0                                     # both
    c.check(c.run(c.step(grad=grad, dw=dw)))


@pytest.mark.parametrize("dv", [False, True])
@pytest.mark.parametrize("dw", [False, True])
def test_rows_outside_the_forms_of_the_scratch_in_one_tile_of_a_pair(dv, dw):
    c = Big(2100, 2048, 32008, 9, seed=41, dv=dv, weights=True, tau=1.5)
    c.W[:, 0] = -6.0
    c.H[:, 0] = 0.0
    for tile, rows in ((1, slice(0, 128, 9)), (2, slice(0, 128)), (6, slice(5, 6)), (7, slice(77, 99)), (16, slice(0, 52, 3))):
        c.H[tile * 128:(tile + 1) * 128, 0][rows] = 10.0      # logits 40 lower: a log-sum-exp near -30
        c.mask[tile * 128:(tile + 1) * 128][rows] = 1
    c.H[10 * 128 + 3, 0] = -14.0                              # and one near 66
    c.mask[10 * 128 + 3] = 1
    st = c.run(c.step(dw=dw))
    # (the norm of dH without its first column: W is constant there, and sum_v g_v w is 0 but for the rounding of the g_v; so leave it out)
    live = c.mask != 0
    assert ((st.lse[live] < -20) | (st.lse[live] > 59)).sum() > 100
    H, W = c.H.double(), c.W.double()
    x = H @ W.t() / c.tau
    p = torch.softmax(x, dim=1)
    r = torch.softmax(c.logits.double() / c.tau, dim=1)
    g = p.scatter_add(1, c.ids.long(), -r) * (torch.where(live, c.weights.double(), 0.0) / c.tau)[:, None]
    dH = g @ W
    for tile in range(0, 2100, 128):
        got, want = st.dH[tile:tile + 128, 1:].double(), dH[tile:tile + 128, 1:]
        assert (got - want).norm() <= TILE_NORM * want.norm(), tile
    assert not st.dH[~live].any() and int(st.status.item()) == 0
    if dw:
        got, want = (st.dW.t() if dv else st.dW).double(), g.t() @ H
        assert (got - want).norm() <= NORM * want.norm()


@pytest.mark.parametrize("dv", [False, True])
def test_several_scratch_passes_of_pairs(dv):
    """A workspace for 2,100 of 4,500 rows at a time: passes of 2,048, 2,048 and 404 rows."""
    c = Big(4500, 2048, 32008, 9, seed=42, dv=dv)
    least = _ais().distill_workspace_min_bytes(c.step(fill=False).shape, 9, _ais().DISTILL_DH)
    row = (32008 + 63) // 64 * 64 * 2
    st = c.step(workspace_bytes_cap=least + (2100 - 128) * row)
    assert (st.workspace.numel() - least) // row == 1972
    c.check(c.run(st))


@pytest.mark.parametrize("dw", [False, True])
def test_results_repeat_bit_for_bit(dw):
    c = Big(2100, 2048, 32008, 17, seed=43)
    st = c.run(c.step(dw=dw))
    outs = lambda: [t.clone() for t in (st.kl, st.lse, st.loss, st.dH) + ((st.dW,) if dw else ())]  # noqa: E731
    first = outs()
    for _ in range(3):
        st.workspace.fill_(255)
        c.run(st)
        assert all(torch.equal(a, b) for a, b in zip(first, outs()))
