"""Timing cases of the operators around on-policy distillation: drawing tokens, a teacher's top logits, the distillation loss.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare(case, seed)`` makes what a program holds
before the call, ``run(state)`` is one pass and ``work(case)`` states the bytes and operations that pass cannot do without.
``exact(case, seed)`` gives the same outputs from the definitions in 64 bits.

Three operations:

  sample   one token per row of logits: temperature, top-k, top-p and min-p, from given uniform numbers, with its log-probs
  top      a teacher's K largest logits per row in order, their ids, and the log-sum-exp of the row
  distill  KL from a teacher's top logits to the softmax of the LM head, its gradient for H and for the head
           (``grad``: 0 the loss alone, 1 with dH, 2 with dH and dW)

``own`` false: plain torch operations; true: the package's entry points.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------------------------------ cases
def _sample(name, rows, V, dtype, how, T=1.0, k=0, p=1.0, m=0.0, banned=False, pad=0):
    return dict(name=name, op="sample", rows=rows, V=V, dtype=dtype, how=how, T=T, k=k, p=p, m=m, banned=banned, pad=pad)


def _top(name, rows, V, dtype, K, tau=1.0, pad=0):
    return dict(name=name, op="top", rows=rows, V=V, dtype=dtype, K=K, tau=tau, pad=pad)


def _distill(name, T, d, V, K, grad, tau=1.0, full=False, dv=False, valid=1.0):
    return dict(name=name, op="distill", T=T, d=d, V=V, K=K, grad=grad, tau=tau, full=full, dv=dv, valid=valid)


def listed():
    return [
        # one sequence decoding: nucleus sampling of a single row, latency counts
        _sample("sample_one_row", 1, 151936, "bf16", "all", T=0.7, p=0.95),
        # a rollout of 8 prompts x 8 responses, one step: plain sampling at temperature 1, as GRPO wants it
        _sample("sample_rollout", 64, 151936, "fp32", "all"),
        # a serving batch whose requests bring their own parameters, some tokens banned
        _sample("sample_mixed_batch", 256, 151936, "bf16", "rows", banned=True),
        # the large-vocabulary head, top-k and min-p, many rows
        _sample("sample_top_k", 512, 262144, "fp16", "all", T=0.8, k=50, m=0.02),
        # a teacher scoring one response
        _top("top_one_response", 613, 151936, "bf16", 64),
        # a chunk of a teacher's logits of the masked-diffusion head, kept in fp32, softened, padded rows
        _top("top_chunk", 2048, 126464, "fp32", 128, tau=2.0, pad=8),
        # the smallest batch, 2 x 4 responses of 64 tokens
        _distill("distill_tiny", 512, 256, 1024, 16, 1),
        # one response: loss and dH
        _distill("distill_one_response", 613, 4096, 151936, 64, 1),
        # a group of responses: loss and dH, softened, rows of padding among them
        _distill("distill_one_group", 9217, 4096, 151936, 64, 1, tau=2.0, valid=0.95),
        # held-out loss against the teacher's own probabilities
        _distill("distill_score", 2048, 4096, 126464, 32, 0, full=True),
        # head stored [d, V], trained itself
        _distill("distill_head_dv", 2305, 4096, 151936, 128, 2, dv=True),
        # scale-block-32 model's wide head, dH and dW
        _distill("distill_large_vocab", 1201, 5120, 262144, 20, 2, full=True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "distill", "distill"])
    if op == "sample":
        V = int(_log(rng, 1000, 262144))
        rows = int(_log(rng, 1, 1024))
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        how = rng.choice(["rows", "all"])
        c = _sample("", rows, V, dtype, how, T=rng.choice([1.0, 0.6, 0.9, 1.3]), k=rng.choice([0, 0, 1, 20, 50, 300, 2000]),
                    p=rng.choice([1.0, 1.0, 0.9, 0.95, 0.5]), m=rng.choice([0.0, 0.0, 0.01, 0.1]), banned=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 1, 8]))
    elif op == "top":
        V = int(_log(rng, 1000, 262144))
        rows = int(_log(rng, 1, min(8192, 5e8 / V)))
        c = _top("", rows, V, rng.choice(["bf16", "fp16", "fp32"]), int(_log(rng, 1, 256)), tau=rng.choice([1.0, 0.5, 2.0]),
                 pad=rng.choice([0, 0, 3, 8]))
    else:
        small = rng.random() < 0.3
        d = 128 * (rng.randint(2, 8) if small else rng.randint(16, 40))
        V = 8 * int(_log(rng, 1024, 16384) / 8) if small else 8 * int(_log(rng, 32000, 262144) / 8)
        grad = rng.choice([0, 1, 1, 2])
        most = 9217.0 * 4096 * 151936 * 2 / (d * V) / (1 + grad)                  # rows at the largest listed case's cost
        T = int(_log(rng, 1, max(2, min(9217, most))))
        c = _distill("", T, d, V, int(_log(rng, 1, 256)), grad, tau=rng.choice([1.0, 0.7, 2.0, 3.0]), full=rng.random() < 0.4,
                     dv=rng.random() < 0.3, valid=rng.choice([1.0, 0.9]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
class _State:
    pass


_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _logits(rows, V, dtype, pad, gen):
    """Rows of an LM's logits: between unsure (standard deviation 1) and confident (6); the last `pad` columns are padding."""
    out = torch.empty(rows, V + pad, dtype=_DTYPES[dtype], device="cuda")
    step = max(1, (1 << 27) // (V + pad))
    for r0 in range(0, rows, step):
        n = min(step, rows - r0)
        sd = 1.0 + 5.0 * torch.rand(n, 1, generator=gen, device="cuda")
        out[r0:r0 + n] = torch.randn(n, V + pad, generator=gen, device="cuda") * sd
    return out[:, :V]


def _hidden(T, d, gen):
    """Hidden states after an RMS norm, of a gain between 1 and 4 (unsure to confident positions), bf16."""
    h = torch.randn(T, d, generator=gen, device="cuda")
    h *= torch.rsqrt(h.pow(2).mean(dim=1, keepdim=True) + 1e-6)
    return (h * (1.0 + 3.0 * torch.rand(T, 1, generator=gen, device="cuda"))).to(torch.bfloat16)


def _head(V, d, gen):
    """LM head, one row per vocabulary entry; logits of unit order at every width."""
    W = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    rows = max(1, (1 << 26) // d)
    for r0 in range(0, V, rows):
        W[r0:r0 + rows] = torch.randn(min(rows, V - r0), d, generator=gen, device="cuda") * (1.28 / math.sqrt(d))
    return W


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = _State()
    s.op = case["op"]
    if s.op in ("sample", "top"):
        rows, V = case["rows"], case["V"]
        s.x = _logits(rows, V, case["dtype"], case["pad"], gen)
        if s.op == "top":
            s.K, s.tau = min(case["K"], V), case["tau"]
            return s
        s.u = torch.rand(rows, generator=gen, device="cuda")
        if case["banned"]:
            ids = torch.randint(0, V, (max(1, V // 100),), generator=gen, device="cuda")
            s.x[:, ids] = -math.inf
        if case["how"] == "rows":
            def pick(values, dtype):
                at = torch.randint(0, len(values), (rows,), generator=gen, device="cuda")
                return torch.tensor(values, dtype=dtype, device="cuda")[at]
            s.T = pick([1.0, 0.7, 0.0, 1.2], torch.float32)
            s.k = pick([0, 0, 40, 1, 500], torch.int32)
            s.p = pick([1.0, 0.95, 0.8], torch.float32)
            s.m = pick([0.0, 0.0, 0.05], torch.float32)
        else:
            s.T, s.k, s.p, s.m = case["T"], case["k"], case["p"], case["m"]
        return s
    T, d, V = case["T"], case["d"], case["V"]
    s.K = min(case["K"], V)
    s.tau, s.dv, s.grad = case["tau"], case["dv"], case["grad"]
    s.H = _hidden(T, d, gen)
    W = _head(V, d, gen)
    # the teacher: the student's logits moved by noise of standard deviation 2, a few units of KL
    s.ids = torch.empty(T, s.K, dtype=torch.int32, device="cuda")
    s.logits = torch.empty(T, s.K, dtype=torch.float32, device="cuda")
    s.lse = torch.empty(T, dtype=torch.float32, device="cuda") if case["full"] else None
    step = max(1, (1 << 28) // V)
    for r0 in range(0, T, step):
        z = (s.H[r0:r0 + step] @ W.t()).float()
        z += 2.0 * torch.randn(z.shape, generator=gen, device="cuda")
        v, i = z.topk(s.K, dim=1)
        s.ids[r0:r0 + step] = i.to(torch.int32)
        s.logits[r0:r0 + step] = v
        if case["full"]:
            s.lse[r0:r0 + step] = torch.logsumexp(z / s.tau, dim=1)
    del z
    s.W = W.t().contiguous() if s.dv else W
    s.mask = (torch.rand(T, generator=gen, device="cuda") < case["valid"]).to(torch.uint8)
    s.mask[0] = 1
    s.step = None
    if own:
        import paper_2605_13907_b200 as ais
        s.step = ais.DistillStep(T, d, V, s.K, temperature=s.tau, want_grad=s.grad > 0, want_dw=s.grad > 1,
                                 w_layout=ais.W_DV if s.dv else ais.W_VD)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        import paper_2605_13907_b200 as ais
        if s.op == "sample":
            r = ais.sample(s.x, s.u, temperature=s.T, top_k=s.k, top_p=s.p, min_p=s.m)
            return dict(tokens=r.tokens, lp=r.lp, lp_full=r.lp_full, n_kept=r.n_kept)
        if s.op == "top":
            r = ais.top_logits(s.x, s.K, temperature=s.tau)
            return dict(ids=r.ids, values=r.values, lse=r.lse)
        st = s.step
        st.step(s.H, s.W, s.ids, s.logits, teacher_lse=s.lse, mask=s.mask)
        out = dict(kl=st.kl, loss=st.loss)
        if s.grad > 0:
            out["dH"] = st.dH
        if s.grad > 1:
            out["dW"] = st.dW
        return out
    return {"sample": _plain_sample, "top": _plain_top, "distill": _plain_distill}[s.op](s)


def _per_row(v, rows, dtype):
    return v.to(dtype)[:, None] if torch.is_tensor(v) else torch.full((rows, 1), v, dtype=dtype, device="cuda")


def _plain_sample(s):
    rows, V = s.x.shape
    T, p, m = (_per_row(v, rows, torch.float32).double() for v in (s.T, s.p, s.m))
    k = _per_row(s.k, rows, torch.int64)
    greedy = T == 0
    T = torch.where(greedy, 1.0, T)
    k = torch.where(greedy, 1, torch.where(k <= 0, V, k))
    x, order = torch.sort(s.x.float(), dim=1, descending=True, stable=True)
    # borders lie within 1e-7 of sums over the vocabulary: masses in 64 bits
    logp = (x.double() - x[:, :1].double()) / T
    e = torch.exp(logp)
    full = e.sum(dim=1)
    first = torch.arange(V, device="cuda")[None, :]
    kept = (first < k) & (x > -math.inf)
    e1 = torch.where(kept, e, 0.0)
    before = torch.cumsum(e1, dim=1) - e1
    kept &= (before < p * e1.sum(dim=1, keepdim=True)) | (p >= 1)
    kept &= e >= m
    kept[:, 0] = True
    w = torch.zeros_like(e).scatter_(1, order, torch.where(kept, e, 0.0))
    mass = torch.cumsum(w, dim=1)
    total = mass[:, -1:]
    token = (mass <= s.u.double()[:, None] * total).sum(dim=1).clamp_(max=V - 1)
    logp = torch.log(w.gather(1, token[:, None])).squeeze(1)
    return dict(tokens=token.to(torch.int32), lp=(logp - torch.log(total.squeeze(1))).float(), lp_full=(logp - torch.log(full)).float(),
                n_kept=kept.sum(dim=1).to(torch.int32))


def _plain_top(s):
    x, order = torch.sort(s.x.float(), dim=1, descending=True, stable=True)
    z = x / s.tau
    lse = z[:, 0] + torch.log(torch.exp(z - z[:, :1]).sum(dim=1))
    return dict(ids=order[:, :s.K].to(torch.int32), values=x[:, :s.K].contiguous(), lse=lse)


def _plain_distill(s):
    W = s.W.float()
    W = W.t() if s.dv else W                                                     # [V, d]
    H = s.H.float()
    x = (H @ W.t()) / s.tau
    top = x.amax(dim=1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    t = s.logits.float() / s.tau
    t_top = t.amax(dim=1, keepdim=True)
    lse_k = t_top + torch.log(torch.exp(t - t_top).sum(dim=1, keepdim=True))
    logr = t - lse_k
    r = torch.exp(logr)
    log_mass = lse_k - s.lse[:, None] if s.lse is not None else torch.zeros_like(lse_k)
    mass = torch.exp(log_mass)
    ids = s.ids.long()
    live = s.mask.float()[:, None]
    weight = live / live.sum()
    kl = (mass * (r * (logr + log_mass - x.gather(1, ids) + lse)).sum(dim=1, keepdim=True) * live).squeeze(1)
    out = dict(kl=kl, loss=(kl * weight.squeeze(1)).sum().reshape(1))
    if s.grad > 0:
        del x
        p.div_(total)
        g = p.scatter_add_(1, ids, -r)
        g *= mass * weight / s.tau
        out["dH"] = (g @ W).to(torch.bfloat16)
        if s.grad > 1:
            dW = g.t() @ H
            out["dW"] = (dW.t() if s.dv else dW).to(torch.bfloat16).contiguous()
    return out


# ------------------------------------------------------------------------------------------ 64 bits, from the definitions
def exact(case, seed):
    if case["op"] == "distill" and (1 + case["grad"]) * 2.0 * case["T"] * case["d"] * case["V"] > 6e13:
        return None
    s = prepare(case, seed)
    if s.op == "distill":
        return _exact_distill(s)
    return _exact_sample(s) if s.op == "sample" else _exact_top(s)


def _exact_sample(s):
    """Row by row, with thresholds on the sorted values; ties at a threshold by a count along the row."""
    rows, V = s.x.shape
    out = dict(tokens=[], lp=[], lp_full=[], n_kept=[])
    at = lambda v, i: float(v[i]) if torch.is_tensor(v) else float(np.float32(v))  # noqa: E731
    for i in range(rows):
        x = s.x[i].double()
        T, k, p, m = at(s.T, i), int(at(s.k, i)), at(s.p, i), at(s.m, i)
        if T == 0:
            T, k = 1.0, 1
        logw = (x - x.max()) / T
        w = torch.exp(logw)
        values = torch.sort(x[x > -math.inf], descending=True).values
        n = values.numel() if k <= 0 else min(k, values.numel())
        ws = torch.exp((values[:n] - values[0]) / T)
        if p < 1:
            cum = torch.cumsum(ws, 0)
            n = min(n, int((cum < p * cum[-1]).sum()) + 1)                      # up to the first that reaches p
        n = max(1, min(n, int((ws[:n] >= m).sum())))
        last = values[n - 1]
        above = x > last
        tie = x == last
        keep = above | (tie & (torch.cumsum(tie.int(), 0) <= n - int(above.sum())))
        cum = torch.cumsum(torch.where(keep, w, 0.0), 0)
        v = int(torch.searchsorted(cum, at(s.u, i) * cum[-1], right=True).clamp_(max=V - 1))
        out["tokens"].append(v)
        out["lp"].append(logw[v] - torch.log(cum[-1]))
        out["lp_full"].append(logw[v] - torch.log(w.sum()))
        out["n_kept"].append(n)
    return dict(tokens=torch.tensor(out["tokens"], dtype=torch.int32), lp=torch.stack(out["lp"]), lp_full=torch.stack(out["lp_full"]),
                n_kept=torch.tensor(out["n_kept"], dtype=torch.int32))


def _exact_top(s):
    """Largest first by repeated selection of chunks of rows in 64 bits: the value and then the smaller index decide."""
    ids, values, lse = [], [], []
    V = s.x.shape[1]
    for part in s.x.split(max(1, (1 << 26) // V)):
        x = part.double()
        # equal values in the order of their indices: topk gives the values, a second sort the places
        v = x.topk(s.K, dim=1).values
        for row, top in zip(x, v):
            where = (row >= top[-1]).nonzero().squeeze(1)
            by_value = torch.sort(row[where], descending=True, stable=True).indices
            ids.append(where[by_value][:s.K].to(torch.int32))
        values.append(v)
        lse.append(torch.logsumexp(x / s.tau, dim=1))
    return dict(ids=torch.stack(ids), values=torch.cat(values), lse=torch.cat(lse))


def _exact_distill(s):
    W = s.W.double()
    if s.dv:
        W = W.t()
    T = s.H.shape[0]
    n = float(s.mask.sum())
    kl, dH = [], []
    dW = torch.zeros_like(W) if s.grad > 1 else None
    step = max(1, (1 << 28) // W.shape[0])
    for r0 in range(0, T, step):
        sl = slice(r0, r0 + step)
        h = s.H[sl].double()
        logp = torch.log_softmax(h @ W.t() / s.tau, dim=1)
        t = s.logits[sl].double() / s.tau
        logq = t - (torch.logsumexp(t, dim=1, keepdim=True) if s.lse is None else s.lse[sl].double()[:, None])
        q = logq.exp()
        ids = s.ids[sl].long()
        live = s.mask[sl].double()
        kl.append((q * (logq - logp.gather(1, ids))).sum(dim=1) * live)
        if s.grad > 0:
            g = logp.exp_() * q.sum(dim=1, keepdim=True)
            g.scatter_add_(1, ids, -q)
            g *= (live / (n * s.tau))[:, None]
            dH.append(g @ W)
            if dW is not None:
                dW += g.t() @ h
    kl = torch.cat(kl)
    out = dict(kl=kl, loss=(kl.sum() / n).reshape(1))
    if s.grad > 0:
        out["dH"] = torch.cat(dH)
    if dW is not None:
        out["dW"] = dW.t().contiguous() if s.dv else dW
    return out


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "distill":
        T, d, V, K, grad = (case[n] for n in ("T", "d", "V", "K", "grad"))
        n = T * case["valid"]
        rows = n * (2.0 * d + 8.0 * min(K, V)) + 5.0 * T + (4.0 * T if case["full"] else 0.0)
        return dict(bytes=2.0 * V * d + rows + (2.0 * T * d if grad > 0 else 0.0) + (2.0 * V * d if grad > 1 else 0.0),
                    flops=2.0 * n * d * V * (1 + grad))
    rows, V = case["rows"], case["V"]
    es = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "top":
        return dict(bytes=rows * (es * V + 8.0 * min(case["K"], V) + 4), flops=2.0 * rows * V)
    return dict(bytes=rows * (es * V + 20.0 + (16.0 if case["how"] == "rows" else 0.0)), flops=2.0 * rows * V)
