"""The distillation step against its float64 definition (GPU).

Tolerances, from the arithmetic.  A logit is a contraction of d terms whose partial sums the tensor core cuts after every 16: off by
at most (d / 16) 2^-23 A / tau, A = max_v sum_i |h_i W_vi| of the row (`dx`; the mean correction is smaller).  The log-sum-exp moves by no
more than its logits, plus its fp32 exponentials and sums: 1.5e-5 as in the sampling tests, e^x in the scratch by 2^-22 + 100 x 2^-24
relative.  So kl: mass (2 dx + 1.5e-5), and 2^-24 of itself for the output.  A scratch entry g is rounded to bf16 once (2^-8 of itself at
most) after an error of p (2 dx + 2e-5) times the row's factor f = |w| mass / tau; the contraction over n terms cuts its partial
sums, (n / 16) 2^-23 of sum |g W|; and dH is rounded once more.  dW likewise over the rows.  With dW the scratch comes from logits in
steps of 1/640, off by 1/1280: another 8e-4 p f (e^(1/1280) - 1 = 7.8e-4).
"""

import numpy as np
import pytest
import torch

from oracle import distill as od

pytestmark = pytest.mark.gpu

STEP16 = 2.0 ** -8
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _ais():
    import paper_2605_13907_b200 as ais
    return ais


def _np(x):
    return x.detach().double().cpu().numpy()


class Case:
    def __init__(self, T, d, V, K, seed, tau=1.0, full=False, weights=False, dv=False, dtype="fp32", masked=0.0, gain=3.0, ldh=None, ldk=None):
        rng = np.random.default_rng(seed)
        self.ldh, self.tau, self.dv = ldh or d, tau, dv
        H = rng.standard_normal((T, d)) * rng.uniform(1.0, gain, (T, 1))
        buf = torch.full((T, self.ldh), float("nan"), dtype=torch.bfloat16)
        buf[:, :d] = torch.from_numpy(H)
        self.H = buf.cuda()[:, :d]
        self.W = torch.from_numpy(rng.standard_normal((V, d)) * (1.28 / np.sqrt(d))).to(torch.bfloat16).cuda()
        z = _np(self.H) @ _np(self.W).T + rng.standard_normal((T, V))
        ids = np.argsort(-z, axis=1)[:, :K]
        t = np.take_along_axis(z, ids, axis=1)
        ldk = ldk or K
        self.ids = torch.full((T, ldk), -5, dtype=torch.int32, device="cuda")[:, :K]
        self.ids.copy_(torch.from_numpy(ids.astype(np.int32)))
        self.logits = torch.full((T, ldk), float("nan"), dtype=DTYPES[dtype], device="cuda")[:, :K]
        self.logits.copy_(torch.from_numpy(t))
        m = z.max(axis=1) / tau
        self.lse = torch.from_numpy(m + np.log(np.exp(z / tau - m[:, None]).sum(axis=1))).float().cuda() if full else None
        self.weights = torch.from_numpy(rng.standard_normal(T)).float().cuda() if weights else None
        mask = (rng.random(T) >= masked).astype(np.uint8)
        mask[T // 2] = 1
        self.mask = torch.from_numpy(mask).cuda()

    def head(self):
        return self.W.t().contiguous() if self.dv else self.W

    def step(self, grad=True, dw=False, **kw):
        T, d = self.H.shape
        ais = _ais()
        return ais.DistillStep(T, d, self.W.shape[0], self.ids.shape[1], temperature=self.tau, want_grad=grad, want_dw=dw, ldh=self.ldh,
                               w_layout=ais.W_DV if self.dv else ais.W_VD, **kw)

    def run(self, st):
        st.step(self.H, self.head(), self.ids, self.logits, teacher_lse=self.lse, mask=self.mask, weights=self.weights)
        torch.cuda.synchronize()
        return st

    def want(self):
        f = lambda a: None if a is None else _np(a)  # noqa: E731
        return od.distill(_np(torch.nan_to_num(self.H)), _np(self.W), self.ids.cpu().numpy(), _np(self.logits), self.mask.cpu().numpy(), self.tau,
                          f(self.lse), f(self.weights))

    def check(self, st, flags=0):
        r = self.want()
        H, W = np.abs(_np(torch.nan_to_num(self.H))), np.abs(_np(self.W))
        T, d = H.shape
        V = W.shape[0]
        dx = (d / 16) * 2.0 ** -23 * (H @ W.T).max(axis=1) / self.tau
        live = self.mask.cpu().numpy() != 0
        n = live.sum()
        w = _np(self.weights) if self.weights is not None else np.full(T, 1.0 / max(n, 1))
        mass = np.ones(T)
        if self.lse is not None:
            t = np.where(self.ids.cpu().numpy() >= 0, _np(self.logits) / self.tau, -np.inf)
            mass = np.exp(t - _np(self.lse)[:, None]).sum(axis=1)
        tol = mass * (2 * dx + 1.5e-5) + 2.0 ** -24 * np.abs(r["kl"])
        kl = _np(st.kl)
        assert (np.abs(kl - r["kl"]) <= tol).all(), np.max(np.abs(kl - r["kl"]) / tol)
        assert not kl[~live].any()
        assert (np.abs(_np(st.lse) - r["lse"]) <= dx + 1.5e-5 + 2.0 ** -24 * np.abs(r["lse"])).all()
        lw = np.where(live, np.abs(w), 0.0)
        assert abs(float(st.loss) - r["loss"]) <= (lw * tol).sum() + 2.0 ** -23 * abs(r["loss"])
        if st.dH is not None or st.dW is not None:
            x = _np(torch.nan_to_num(self.H)) @ _np(self.W).T / self.tau
            p = np.exp(x - x.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            code = 8e-4 if st.dW is not None else 0.0
            dg = STEP16 * np.abs(r["g"]) + p * ((2 * dx + 2e-5 + code) * lw * mass / self.tau)[:, None]
        if st.dH is not None:
            tol = dg @ W + (V / 16 + 1) * 2.0 ** -23 * (np.abs(r["g"]) @ W) + 2.0 ** -23 * (p @ W) * (lw * mass / self.tau)[:, None]
            tol += STEP16 * (np.abs(r["dH"]) + tol) + 1e-38
            dH = _np(st.dH)
            assert (np.abs(dH - r["dH"]) <= tol).all(), np.max(np.abs(dH - r["dH"]) / tol)
            assert not dH[~live].any()
            # by norm, too, over the columns in which the head's rows differ: with a constant w, sum_v g_v w is w sum_v g_v, which is (p sums
            # to 1, r to 1) exactly 0, and all that is left of it is the rounding of the g_v, 2^-8 |g_v w| each, which `tol` allows
            cols = W.std(axis=0) > 0
            if np.linalg.norm(r["dH"][:, cols]) > 0:
                assert np.linalg.norm((dH - r["dH"])[:, cols]) <= 5e-3 * np.linalg.norm(r["dH"][:, cols])
        if st.dW is not None:
            tol = dg.T @ H + (T / 16 + 1) * 2.0 ** -23 * (np.abs(r["g"]).T @ H)
            tol += STEP16 * (np.abs(r["dW"]) + tol) + 1e-38
            dW = _np(st.dW).T if self.dv else _np(st.dW)
            assert (np.abs(dW - r["dW"]) <= tol).all(), np.max(np.abs(dW - r["dW"]) / tol)
        assert int(st.status.item()) == flags
        return r


@pytest.mark.parametrize("T,d,V,K", [(1, 128, 8, 1), (1, 256, 1024, 16), (5, 128, 264, 264), (129, 256, 1000, 7), (300, 384, 4104, 33), (513, 256, 1024, 64),
                                     (2, 512, 20000, 1024)])
@pytest.mark.parametrize("dv", [False, True])
@pytest.mark.parametrize("dw", [False, True])
def test_sizes_layouts_and_gradients(T, d, V, K, dv, dw):
    c = Case(T, d, V, K, seed=T + K, dv=dv, masked=0.1)
    c.check(c.run(c.step(dw=dw)))


@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("weights", [False, True])
def test_temperature_mass_and_weights(tau, full, weights):
    for dw in (False, True):
        c = Case(140, 256, 1336, 20, seed=4, tau=tau, full=full, weights=weights, masked=0.2, dtype="bf16" if full else "fp16")
        if full:
            c.lse += 0.5                                      # (bf16 entries may add up to more than their sum before rounding)
        c.check(c.run(c.step(dw=dw)))


def test_loss_alone_and_dw_alone():
    c = Case(200, 256, 2048, 32, seed=5, masked=0.3)
    both = c.run(c.step(dw=True))
    alone = c.run(c.step(grad=False))
    c.check(alone)
    assert torch.equal(alone.kl, both.kl) and torch.equal(alone.loss, both.loss)
    only_dw = c.run(c.step(grad=False, dw=True))
    c.check(only_dw)
    assert only_dw.dH is None and torch.equal(only_dw.dW, both.dW)


def test_gradient_against_differences_of_the_loss():
    """dH and dW in a direction each against central differences of the definition's loss: the gradient's own error (5e-3 of its norm)
    along a unit direction, and h^2 times a third derivative of order one."""
    c = Case(24, 128, 520, 12, seed=6, weights=True, tau=1.5)
    st = c.run(c.step(dw=True))
    rng = np.random.default_rng(7)
    H, W, h = _np(c.H), _np(c.W), 1e-4
    loss = lambda H, W: od.distill(H, W, c.ids.cpu().numpy(), _np(c.logits), np.ones(24) * c.mask.cpu().numpy(), c.tau, None, _np(c.weights))["loss"]  # noqa: E731
    for grad, a, move in ((_np(st.dH), H, lambda D: (H + D, W)), (_np(st.dW), W, lambda D: (H, W + D))):
        D = rng.standard_normal(a.shape)
        D /= np.linalg.norm(D)
        D += grad / np.linalg.norm(grad)                      # (a random direction alone is nearly orthogonal to the gradient)
        num = (loss(*move(h * D)) - loss(*move(-h * D))) / (2 * h)
        assert abs(num - (grad * D).sum()) <= 2 * 5e-3 * np.linalg.norm(grad)


def test_entries_that_count_for_nothing_and_ids_given_twice():
    ais = _ais()
    for dw in (False, True):
        c = Case(150, 256, 1024, 24, seed=8, masked=0.1)
        rng = np.random.default_rng(9)
        ids, t = c.ids.cpu().numpy().copy(), _np(c.logits)
        ids[rng.random(ids.shape) < 0.2] = -1
        ids[3] = -1                                           # no entry at all
        t[4] = -np.inf                                        # no probability anywhere
        t[5, ::2] = -np.inf
        ids[6, :12] = ids[6, 12]                              # one id thirteen times
        ids[7] = ids[7, 0]
        ids[8, 3] = ids[8, 4]
        c.mask[3:9] = 1
        c.ids.copy_(torch.from_numpy(ids))
        c.logits.copy_(torch.from_numpy(t))
        st = c.run(c.step(dw=dw))
        c.check(st)
        assert float(st.kl[3]) == 0 and float(st.kl[4]) == 0 and not st.dH[3].any() and not st.dH[4].any()
        ids[10, 2], ids[11, 0] = 1024, 2 ** 31 - 1            # beyond the vocabulary
        c.mask[10:12] = 1
        c.ids.copy_(torch.from_numpy(ids))
        c.check(c.run(c.step(dw=dw)), flags=ais.FLAG_TOKEN_RANGE)


def test_non_finite_rows_leave_the_others_alone():
    ais = _ais()
    for dw in (False, True):
        c = Case(200, 256, 1024, 8, seed=10, weights=True)
        clean = c.run(c.step(dw=dw))
        c.weights[[3, 50, 51, 199]] = 0.0                     # what the marked rows come down to, for dW
        quiet = c.run(c.step(dw=dw))
        c.H[3, 5] = float("nan")
        c.H[50] = float("inf")
        c.logits[51, 2] = float("nan")
        c.logits[199, 0] = float("inf")
        st = c.run(c.step(dw=dw))
        keep = torch.ones(200, dtype=torch.bool, device="cuda")
        keep[[3, 50, 51, 199]] = False
        assert torch.equal(st.kl[keep], clean.kl[keep]) and torch.equal(st.dH[keep], clean.dH[keep])
        assert not st.kl[~keep].any() and not st.dH[~keep].any() and torch.isnan(st.lse[~keep]).all()
        assert int(st.status.item()) == ais.FLAG_NONFINITE
        if dw:
            assert torch.equal(st.dW, quiet.dW)


def test_masked_rows_may_hold_anything():
    c = Case(260, 256, 1024, 8, seed=11, masked=0.5)
    for dw in (False, True):
        clean = c.run(c.step(dw=dw))
        d = Case(260, 256, 1024, 8, seed=11, masked=0.5)
        off = d.mask == 0
        d.H[off] = float("nan")
        d.logits[off] = float("nan")
        d.ids[off] = 1 << 30
        got = d.run(d.step(dw=dw))
        assert torch.equal(got.kl, clean.kl) and torch.equal(got.dH, clean.dH) and int(got.status.item()) == 0
        if dw:
            assert torch.equal(got.dW, clean.dW)


def test_no_valid_row():
    ais = _ais()
    for dw in (False, True):
        c = Case(130, 128, 512, 4, seed=12)
        c.mask.zero_()
        st = c.run(c.step(dw=dw))
        assert float(st.loss) == 0 and not st.kl.any() and not st.dH.any() and (not dw or not st.dW.any())
        assert int(st.status.item()) == ais.FLAG_EMPTY


def test_no_rows_at_all():
    ais = _ais()
    st = ais.DistillStep(0, 128, 512, 4, want_dw=True)
    st.loss.fill_(3.0)
    st.dW.fill_(3.0)
    W = torch.zeros(512, 128, dtype=torch.bfloat16, device="cuda")
    st.step(torch.zeros(0, 128, dtype=torch.bfloat16, device="cuda"), W, torch.zeros(0, 4, dtype=torch.int32, device="cuda"),
            torch.zeros(0, 4, device="cuda"))
    assert float(st.loss) == 0 and not st.dW.any()


@pytest.mark.parametrize("gain", [40.0, 0.0])
def test_rows_outside_the_exponent_form(gain):
    """Log-sum-exps far above the range in which the scratch keeps e^x (gain 40: logits of +-200), and all logits shifted far below."""
    for dv in (False, True):
        c = Case(300, 256, 1024, 12, seed=13, dv=dv, gain=max(gain, 1.0))
        if gain == 0.0:
            # every logit near -60: a hidden unit of 10 that meets -6 in every row of the head, in half of the rows
            c.W[:, 0] = -6.0
            c.H[:, 0] = 0.0
            c.H[::2, 0] = 10.0
        r = c.check(c.run(c.step()))
        assert ((r["lse"] > 59) | (r["lse"] < -20)).sum() > 50
        c.check(c.run(c.step(dw=True)))


def test_strides_and_passes_of_few_rows():
    """Row strides of H / dH and of the teacher; a workspace that holds 128 rows of scratch at a time."""
    ais = _ais()
    c = Case(700, 256, 1024, 10, seed=14, ldh=288, ldk=13, masked=0.2)
    st = c.step()
    want = c.run(st)
    c.check(want)
    small = c.step(workspace_bytes_cap=1)
    assert small.workspace.numel() == ais.distill_workspace_min_bytes(small.shape, 10, ais.DISTILL_DH) < st.workspace.numel()
    c.check(c.run(small))
    # rows with a log-sum-exp outside the exponent form in some of the passes only
    c.H[::97] *= 64.0
    c.check(c.run(small))


def test_results_do_not_depend_on_what_ran_before_and_repeat_bit_for_bit():
    c = Case(400, 256, 2048, 16, seed=15)
    st = c.run(c.step())
    first = [t.clone() for t in (st.kl, st.lse, st.loss, st.dH)]
    other = Case(400, 256, 2048, 16, seed=16, gain=40.0)
    other.run(st)
    st.workspace.fill_(255)                                   # NaNs everywhere
    c.run(st)
    assert all(torch.equal(a, b) for a, b in zip(first, (st.kl, st.lse, st.loss, st.dH)))


def test_streams_and_captured_graphs():
    c = Case(333, 256, 1024, 16, seed=17)
    st = c.run(c.step(dw=True))
    want = [t.clone() for t in (st.kl, st.loss, st.dH, st.dW)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.step(c.H, c.head(), c.ids, c.logits, mask=c.mask)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (st.kl, st.loss, st.dH, st.dW)))
    W = c.head()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.step(c.H, W, c.ids, c.logits, mask=c.mask)
    other = Case(333, 256, 1024, 16, seed=18)
    keep = [t.clone() for t in (c.H, c.ids, c.logits)]
    for src in ((other.H, other.ids, other.logits), keep):
        for dst, s in zip((c.H, c.ids, c.logits), src):
            dst.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (st.kl, st.loss, st.dH, st.dW)))


def test_writes_stay_inside_the_buffers():
    """Outputs and a workspace of the least size, each inside a larger buffer of known bytes; rows of dH and dW with padding between."""
    ais = _ais()
    for dv in (False, True):
        c = Case(150, 256, 1000, 9, seed=21, dv=dv, masked=0.2, ldh=272)
        want = c.run(c.step(dw=True))

        def inside(shape, dtype, pad=0):
            n = int(np.prod(shape[:-1])) * (shape[-1] + pad)
            es = torch.empty(0, dtype=dtype).element_size()
            raw = torch.full((512 + n * es + 512,), 0x5A, dtype=torch.uint8, device="cuda")
            return raw, raw[512:512 + n * es].view(dtype).view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]

        T, d, V = 150, 256, 1000
        raws, out = zip(*(inside((T,), torch.float32), inside((T,), torch.float32), inside((1,), torch.float32), inside((T, d), torch.bfloat16, 16),
                          inside((d, V) if dv else (V, d), torch.bfloat16, 24)))
        size = ais.distill_workspace_min_bytes(want.shape, 9, ais.DISTILL_DH | ais.DISTILL_DW)
        ws_raw, ws = inside((size,), torch.uint8)
        kl, lse, loss, dH, dW = out
        ais.distill(want.shape, c.H, c.head(), c.ids, c.logits, c.mask, kl, loss, ws, lse=lse, dH=dH, dW=dW)
        torch.cuda.synchronize()
        for got, ref in zip(out, (want.kl, want.lse, want.loss, want.dH, want.dW)):
            assert torch.equal(got, ref)
        for raw in raws + (ws_raw,):
            assert (raw[:512] == 0x5A).all() and (raw[-512:] == 0x5A).all()
        for raw, rows, cols, pad in ((raws[3], T, d, 16), (raws[4], d if dv else V, V if dv else d, 24)):
            body = raw[512:-512].view(rows, (cols + pad) * 2)[:, cols * 2:]
            assert (body == 0x5A).all()


def test_refusals_of_the_python_layer():
    ais = _ais()
    c = Case(10, 128, 512, 4, seed=19)
    st = c.step()
    bad = [dict(ids=c.ids.long()), dict(ids=c.ids[:, :3]), dict(logits=c.logits[:5]), dict(H=c.H.float()), dict(W=c.W[:500]), dict(mask=c.mask[:9]),
           dict(weights=torch.ones(10, dtype=torch.float64, device="cuda")), dict(teacher_lse=torch.ones(11, device="cuda")), dict(H=c.H.cpu())]
    for kw in bad:
        a = dict(H=c.H, W=c.W, ids=c.ids, logits=c.logits) | kw
        with pytest.raises(ais.AisError):
            st.step(**a)
    st.step(c.H, c.W, c.ids, c.logits)
    torch.cuda.synchronize()


def test_on_policy_distillation_run():
    """The operators together: logits of a rollout -> tokens and lp_roll; a teacher's logits -> its top entries; hidden states and
    head -> loss and gradients; the tokens and lp_roll go through the GRPO diagnostics."""
    ais = _ais()
    T, d, V, K = 256, 256, 1024, 32
    rng = np.random.default_rng(20)
    H = torch.from_numpy(rng.standard_normal((T, d))).to(torch.bfloat16).cuda()
    W = torch.from_numpy(rng.standard_normal((V, d)) / 16).to(torch.bfloat16).cuda()
    W_teacher = (W.float() + 0.02 * torch.from_numpy(rng.standard_normal((V, d))).float().cuda()).to(torch.bfloat16)
    u = torch.from_numpy(rng.random(T, dtype=np.float32)).cuda()
    drawn = ais.sample((H @ W.t()).float(), u)
    assert (drawn.n_kept == V).all() and float((drawn.lp - drawn.lp_full).abs().max()) <= 1.5e-5
    step = ais.AisStep(T, d, V, 2, 4, 128)
    offsets = torch.arange(0, T + 1, T // 8, dtype=torch.int32, device="cuda")
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    rewards = torch.tensor([1.0, 0, 0, 1, 0, 1, 1, 0], device="cuda")
    step.forward(H, W, drawn.tokens, mask)
    # lp of the sampled tokens: logits rounded to bf16 by the matrix product (2^-8 of up to 8), against the fused pass
    assert float((step.lp_train - drawn.lp).abs().max()) <= 2 * 8 * 2.0 ** -8
    step.lp_roll.copy_(drawn.lp)
    step.diagnose(mask, offsets, rewards)
    assert step.read_diag()["n_valid"] == T and int(step.status.item()) == 0
    top = ais.top_logits((H @ W_teacher.t()).float(), K)
    st = ais.DistillStep(T, d, V, K, want_dw=True)
    st.step(H, W, top.ids, top.values, teacher_lse=top.lse, mask=mask)
    want = od.distill(_np(H), _np(W), top.ids.cpu().numpy(), _np(top.values), np.ones(T), 1.0, _np(top.lse))
    assert abs(float(st.loss) - want["loss"]) <= 1e-4
    assert np.linalg.norm(_np(st.dH) - want["dH"]) <= 5e-3 * np.linalg.norm(want["dH"])
    assert np.linalg.norm(_np(st.dW) - want["dW"]) <= 5e-3 * np.linalg.norm(want["dW"])
