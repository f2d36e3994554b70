"""What sampling, top logits and distillation refuse before any device call, and the sizes of their workspaces (CPU)."""

import ctypes as C

import pytest
import torch

OK, NULL, SHAPE, ALIGN, WORKSPACE, DEVICE, PARAM, LIMIT = 0, -1, -2, -3, -4, -5, -6, -7
P = C.c_void_p(1 << 20)                       # never dereferenced: every call here is refused first


def _lib():
    import paper_2605_13907_b200 as ais
    return ais.lib()


def _how(**kw):
    import paper_2605_13907_b200 as ais
    how = ais.Sampling()
    _lib().ais_default_sampling(C.byref(how))
    for k, v in kw.items():
        setattr(how, k, v)
    return how


def _sample(x=P, dtype=0, rows=4, V=100, ld=100, how=None, u=P, tokens=P):
    return _lib().ais_sample(x, dtype, rows, V, ld, C.byref(how or _how()), u, None, tokens, None, None, None, None, None)


def test_default_sampling():
    how = _how()
    assert (how.temperature, how.top_k, how.top_p, how.min_p) == (1.0, 0, 1.0, 0.0) and not how.temperature_rows


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), PARAM), (dict(dtype=-1), PARAM), (dict(rows=-1), SHAPE), (dict(V=0), SHAPE), (dict(ld=99), SHAPE),
    (dict(V=327681, ld=327681), LIMIT), (dict(rows=(1 << 24) + 1), LIMIT), (dict(x=None), NULL), (dict(u=None), NULL), (dict(tokens=None), NULL),
    (dict(x=C.c_void_p((1 << 20) + 1)), ALIGN), (dict(x=C.c_void_p((1 << 20) + 2), dtype=2), ALIGN)])
def test_sample_refuses(kw, want):
    assert _sample(**kw) == want


@pytest.mark.parametrize("kw", [dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-7),
                                dict(top_p=-0.1), dict(top_p=float("nan")), dict(min_p=1.5), dict(min_p=float("nan"))])
def test_sample_refuses_parameters(kw):
    assert _sample(how=_how(**kw)) == PARAM


def test_null_how_is_refused():
    assert _lib().ais_sample(P, 0, 1, 8, 8, None, P, None, P, None, None, None, None, None) == NULL


@pytest.mark.parametrize("kw,want", [(dict(K=0), SHAPE), (dict(K=101), SHAPE), (dict(K=1025, V=2000, ld=2000, ld_out=2000), LIMIT), (dict(ld_out=4), SHAPE),
                                     (dict(tau=0.0), PARAM), (dict(tau=float("nan")), PARAM), (dict(ids=None), NULL), (dict(values=None), NULL)])
def test_top_logits_refuses(kw, want):
    a = dict(K=5, V=100, ld=100, ld_out=5, tau=1.0, ids=P, values=P) | kw
    assert _lib().ais_top_logits(P, 2, 4, a["V"], a["ld"], a["K"], a["tau"], None, a["ids"], a["values"], a["ld_out"], None, None, None) == want


def _distill(**kw):
    import paper_2605_13907_b200 as ais
    a = dict(T=10, d=128, V=512, K=4, H=P, W=P, ids=P, logits=P, dtype=2, ldk=4, tau=1.0, mask=P, kl=P, dH=None, dW=None, lddw=0, ws=P, bytes=1 << 40,
             layout=0) | kw
    shape = ais.make_shape(a["T"], a["d"], a["V"], 1, 1, 128, w_layout=a["layout"])
    return _lib().ais_distill(C.byref(shape), a["H"], a["W"], a["K"], a["ids"], a["logits"], a["dtype"], a["ldk"], None, a["tau"], a["mask"], None,
                              a["kl"], None, None, a["dH"], a["dW"], a["lddw"], None, a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(K=0), SHAPE), (dict(K=513), SHAPE), (dict(K=1025, V=2048, ldk=1025), LIMIT), (dict(d=100), SHAPE), (dict(V=510), SHAPE), (dict(T=-1), SHAPE),
    (dict(ldk=3), SHAPE), (dict(dtype=4), PARAM), (dict(tau=0.0), PARAM), (dict(tau=-1.0), PARAM), (dict(tau=float("nan")), PARAM),
    (dict(H=None), NULL), (dict(W=None), NULL), (dict(ids=None), NULL), (dict(logits=None), NULL), (dict(mask=None), NULL), (dict(kl=None), NULL),
    (dict(H=C.c_void_p((1 << 20) + 8)), ALIGN), (dict(dH=C.c_void_p((1 << 20) + 8)), ALIGN), (dict(dW=P, lddw=127), SHAPE), (dict(dW=P, lddw=132), ALIGN),
    (dict(dW=P, lddw=128, layout=1), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws=C.c_void_p((1 << 20) + 128)), WORKSPACE), (dict(bytes=4096), WORKSPACE)])
def test_distill_refuses(kw, want):
    assert _distill(**kw) == want


def test_distill_workspace_sizes():
    import paper_2605_13907_b200 as ais
    at = lambda T, g, f=ais.distill_workspace_min_bytes, K=64: f(ais.make_shape(T, 4096, 151936, 3, 7, 0), K, g)  # noqa: E731
    assert at(5, 0) > 0 and at(5, 4) == 0 and at(5, 1, K=1025) == 0 and at(5, 1, K=0) == 0
    for grads in (0, 1, 2, 3):
        sizes = [at(T, grads) for T in list(range(0, 1500, 41)) + [4000, 9217, 40000, 70811]]
        assert sizes == sorted(sizes)                                       # a workspace for the largest batch serves the shorter ones
        rec = [at(T, grads, ais.distill_workspace_bytes) for T in (0, 100, 5000, 70811)]
        assert rec == sorted(rec) and all(r >= at(T, grads) for r, T in zip(rec, (0, 100, 5000, 70811)))
    # one byte less than the minimum is refused, the minimum goes on to the device
    shape = ais.make_shape(10, 128, 512, 1, 1, 128)
    for dH, dW, grads in ((None, None, 0), (P, None, 1), (None, P, 2), (P, P, 3)):
        least = ais.distill_workspace_min_bytes(shape, 4, grads)
        assert _distill(dH=dH, dW=dW, lddw=128, bytes=least - 1) == WORKSPACE
        if not torch.cuda.is_available():
            assert _distill(dH=dH, dW=dW, lddw=128, bytes=least) == DEVICE


def test_python_layer_refuses_cpu_tensors():
    import paper_2605_13907_b200 as ais
    x, u = torch.zeros(2, 8), torch.zeros(2)
    with pytest.raises(ais.AisError):
        ais.sample(x, u)
    with pytest.raises(ais.AisError):
        ais.top_logits(x, 2)
