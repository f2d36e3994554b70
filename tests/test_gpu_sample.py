"""Sampling and top logits against their float64 definitions (GPU).

Tokens, counts and ids have to be equal: the inputs are fixed, and the definition's `margin` says that no row's decision lies within
1e-10 of a border (the kernel's sums are good to 1e-11).  Log-probs: 2^-24 of the value for the rounding of the output; lp_full and lse
come from fp32 exponentials: ex2.approx 2^-22, its argument (2^-24 of at most 64 units of log2, twice rounded) 128 x 2^-24 x ln 2, and a
thread's running sum of at most 128 terms 128 x 2^-24, together below 240 x 2^-24 = 1.5e-5.  lp comes from fp64.
"""

import numpy as np
import pytest
import torch

from oracle import select as osel

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF_STEP = 2.0 ** -24
FULL = 1.5e-5


def _ais():
    import paper_2605_13907_b200 as ais
    return ais


def _logits(rows, V, dtype, seed, scale=(1.0, 6.0), ld=None, lead=0):
    """[rows, V] on the GPU inside a buffer of row stride ld that starts `lead` elements late, everything else NaN."""
    rng = np.random.default_rng(seed)
    ld = ld or V
    x = rng.standard_normal((rows, V)) * rng.uniform(*scale, size=(rows, 1))
    buf = torch.full((lead + rows * ld + 16,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = buf[lead:lead + rows * ld].view(rows, ld)[:, :V]
    view.copy_(torch.from_numpy(x))
    return view


def _u(rows, seed):
    return torch.from_numpy(np.random.default_rng(seed).random(rows, dtype=np.float32)).cuda()


def _np(x):
    return x.detach().double().cpu().numpy()


def _check(x, u, r, status, margin=1e-10, flags=0, **how):
    """`how`: numbers or per-row lists."""
    xs, us = _np(x), _np(u)
    for i in range(x.shape[0]):
        one = {k: (v[i] if np.ndim(v) else v) for k, v in how.items()}
        token, lp, full, n, m = osel.sample_row(xs[i], us[i], **one)
        # (entries of one value only: every sum is a whole number of times its exponential, 1, in both, so a border is exact as well)
        finite = xs[i][np.isfinite(xs[i])]
        assert m > margin or (finite == finite[0]).all(), f"row {i}: a decision lies on a border"
        assert int(r.tokens[i]) == token and int(r.n_kept[i]) == n, (i, one, int(r.tokens[i]), token, int(r.n_kept[i]), n)
        assert abs(float(r.lp[i]) - lp) <= HALF_STEP * abs(lp) + 1e-10
        assert abs(float(r.lp_full[i]) - full) <= HALF_STEP * abs(full) + FULL
    assert int(status.item()) == flags


def _sample(x, u, **how):
    ais = _ais()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    as_row = {k: (torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") if np.ndim(v) else v) for k, v in how.items()}
    r = ais.sample(x, u, status=status, **as_row)
    torch.cuda.synchronize()
    return r, status


HOW = [dict(), dict(temperature=0.7, top_p=0.9), dict(top_k=5), dict(top_k=50, top_p=0.8, min_p=0.05), dict(min_p=0.02, temperature=1.3),
       dict(top_k=1500, top_p=0.95), dict(temperature=0.0), dict(top_p=0.0), dict(top_k=1), dict(top_p=0.999, temperature=2.0)]


@pytest.mark.parametrize("how", HOW, ids=str)
@pytest.mark.parametrize("V", [1, 2, 31, 1000, 4097, 151936])
def test_sizes_and_filters(V, how):
    for dtype in DTYPES:
        x = _logits(3, V, dtype, V)
        u = _u(3, V + 1)
        _check(x, u, *_sample(x, u, **how), **how)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lead,pad", [(0, 0), (1, 0), (3, 5), (8, 1), (0, 8)])
def test_strides_and_alignment(dtype, lead, pad):
    V = 20011
    x = _logits(5, V, dtype, lead + pad, ld=V + pad, lead=lead)
    u = _u(5, 1)
    for how in (dict(top_p=0.9), dict(top_k=40)):
        _check(x, u, *_sample(x, u, **how), **how)


@pytest.mark.parametrize("rows", [1, 2, 37, 150, 600])
def test_row_counts_and_parameters_of_their_own(rows):
    rng = np.random.default_rng(rows)
    x, u = _logits(rows, 5003, "bf16", rows), _u(rows, rows)
    how = dict(temperature=rng.choice([0.0, 0.5, 1.0, 3.0], rows), top_k=rng.choice([-1, 0, 1, 7, 400, 1500, 9999], rows),
               top_p=rng.choice([0.3, 0.9, 1.0, 2.0], rows), min_p=rng.choice([-1.0, 0.0, 0.1, 1.0], rows))
    _check(x, u, *_sample(x, u, **how), **how)


@pytest.mark.parametrize("V", [4099, 151936])
@pytest.mark.parametrize("levels", [1, 2, 30])
def test_equal_values(V, levels):
    """Thousands of entries share a value: which ones are kept goes by index, and a cut lies inside such a group."""
    rng = np.random.default_rng(levels)
    x = torch.from_numpy(rng.integers(0, levels, (4, V)) / 4.0 - 3.0).to(torch.bfloat16).cuda()
    u = _u(4, V)
    for how in (dict(top_k=7), dict(top_k=1024), dict(top_k=3333), dict(top_p=0.37), dict(top_k=3333, top_p=0.61), dict(min_p=1.0), dict()):
        # sums of equal terms sit 1 / V from their borders
        _check(x, u, *_sample(x, u, **how), margin=1e-12, **how)


def test_borders_of_u_are_exact():
    """All entries equal: the token is floor(u V), at u = k / V exactly and one step below."""
    V = 1024
    k = np.array([0, 1, 511, 512, 1023])
    u = np.concatenate([k / V, np.nextafter(np.float32(k[1:] / V), np.float32(0)), [np.nextafter(np.float32(1), np.float32(0))]]).astype(np.float32)
    x = torch.zeros(len(u), V, device="cuda")
    r, status = _sample(x, torch.from_numpy(u).cuda())
    assert r.tokens.tolist() == [0, 1, 511, 512, 1023, 0, 510, 511, 1022, 1023] and int(status.item()) == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_entries(dtype):
    """-inf and the type's lowest value in masked places; rows that keep one entry, or none."""
    V = 9001
    x = _logits(8, V, dtype, 5)
    rng = np.random.default_rng(6)
    low = torch.finfo(DTYPES[dtype]).min
    for i, v in enumerate([-np.inf, low, -np.inf, low]):
        x[i, torch.from_numpy(rng.permutation(V)[:V - 40]).cuda()] = v
    x[4] = -np.inf
    x[4, 4321] = -7.0
    x[5] = low
    x[6] = -np.inf
    u = _u(8, 7)
    for how in (dict(), dict(top_p=0.9), dict(top_k=64), dict(top_k=60, top_p=0.5, min_p=0.1), dict(top_k=2000)):
        r, status = _sample(x, u, **how)
        _check(x, u, r, status, margin=1e-12, flags=_ais().FLAG_EMPTY, **how)
        assert int(r.tokens[6]) == -1 and float(r.lp[6]) == 0.0 and int(r.n_kept[6]) == 0


def test_degenerate_scales():
    """Logits that leave the histogram's range, fall into one bin of it, or differ by single steps of fp32."""
    rng = np.random.default_rng(8)
    V = 30011
    rows = [rng.standard_normal(V) * 1e4, rng.standard_normal(V) * 1e-3, 1.0 + np.arange(V) * 2.0 ** -23, rng.standard_normal(V) * 1e30,
            -np.abs(rng.standard_normal(V)) * 1e-30, np.where(rng.random(V) < 0.5, 0.0, -0.0)]
    x = torch.from_numpy(np.stack(rows)).float().cuda()
    u = _u(len(rows), 9)
    for how in (dict(), dict(top_k=30), dict(top_k=1024, top_p=0.7), dict(top_k=5000, top_p=0.7), dict(top_p=0.4), dict(temperature=1e-6, top_k=30),
                dict(temperature=1e6, top_p=0.5), dict(temperature=50.0, top_k=2500)):
        _check(x, u, *_sample(x, u, **how), margin=1e-12, **how)


def test_bad_rows_and_masked_rows_are_refused_alone():
    ais = _ais()
    V = 3001
    x = _logits(9, V, "fp32", 10)
    x[1, 17] = float("nan")
    x[2, 2999] = float("inf")
    u = _u(9, 11)
    u[3] = 1.0
    u[4] = float("nan")
    mask = torch.ones(9, dtype=torch.uint8, device="cuda")
    mask[5] = 0
    T = torch.ones(9, device="cuda")
    T[6] = -1.0
    T[7] = 1e-7
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = ais.sample(x, u, temperature=T, top_p=0.9, mask=mask, status=status)
    assert r.tokens[1:8].tolist() == [-1] * 7 and not r.lp[1:8].any() and not r.lp_full[1:8].any() and not r.n_kept[1:8].any()
    assert int(status.item()) == ais.FLAG_NONFINITE | ais.FLAG_PARAM
    status.zero_()
    _check(x[[0, 8]], u[[0, 8]], ais.Sampled(*(t[[0, 8]] for t in r)), status, top_p=0.9)


def test_rows_behind_the_last_are_left_alone_and_calls_are_independent():
    """Outputs given by the caller; a row alone and among others draws the same token with the same bits."""
    ais = _ais()
    x, u = _logits(40, 151936, "bf16", 12), _u(40, 13)
    out = ais.Sampled(*(torch.full((64,), 77, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.float32, torch.int32)))
    ais.sample(x, u, top_p=0.8, out=ais.Sampled(*(t[:40] for t in out)))
    for t in out:
        assert (t[40:] == 77).all()
    for i in (0, 39):
        r = ais.sample(x[i:i + 1], u[i:i + 1], top_p=0.8)
        for a, b in zip(r, out):
            assert float(a[0]) == pytest.approx(float(b[i]), abs=2e-6)
        assert int(r.tokens[0]) == int(out.tokens[i])
    again = ais.sample(x, u, top_p=0.8)
    assert all(torch.equal(a, b[:40]) for a, b in zip(again, out))


def test_streams_and_captured_graphs():
    ais = _ais()
    x, u = _logits(16, 50003, "fp32", 14), _u(16, 15)
    want = ais.sample(x, u, top_k=50, top_p=0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ais.sample(x, u, top_k=50, top_p=0.9)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = ais.Sampled(*(torch.zeros_like(t) for t in want))
    x2, u2 = _logits(16, 50003, "fp32", 16), _u(16, 17)
    static_x, static_u = x.clone(), u.clone()
    ais.sample(static_x, static_u, top_k=50, top_p=0.9, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ais.sample(static_x, static_u, top_k=50, top_p=0.9, out=out)
    for a, b in ((x2, u2), (x, u)):
        static_x.copy_(a)
        static_u.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, ais.sample(a, b, top_k=50, top_p=0.9)))


def test_captured_with_parameters_of_their_own_behind_a_kernel_that_writes_them():
    """Two launches that overlap: both see what the kernels before them wrote, and the kernel behind them sees both."""
    ais = _ais()
    rows, V = 300, 20011
    x, u = _logits(rows, V, "bf16", 30), _u(rows, 31)
    rng = np.random.default_rng(32)
    k = torch.from_numpy(rng.choice([0, 5, 2000], rows).astype(np.int32)).cuda()
    p = torch.from_numpy(rng.choice([0.5, 0.9, 1.0], rows).astype(np.float32)).cuda()
    src = torch.empty_like(x)
    out = ais.Sampled(*(torch.zeros(rows, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.float32, torch.int32)))
    seen = torch.zeros(rows, dtype=torch.int32, device="cuda")

    def go():
        src.copy_(x)
        ais.sample(src, u, top_k=k, top_p=p, out=out)
        seen.copy_(out.tokens)
        src.zero_()

    go()
    torch.cuda.synchronize()
    want = seen.clone()
    _check(x, u, out, torch.zeros(1, dtype=torch.int32), top_k=k.tolist(), top_p=p.tolist())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            go()
    for _ in range(5):
        seen.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(seen, want)


def test_two_streams_at_once():
    ais = _ais()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    x, u = _logits(64, 50003, "fp32", 33), _u(64, 34)
    want = ais.sample(x, u, top_p=0.9), ais.top_logits(x, 50)
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        with torch.cuda.stream(a):
            got.append((ais.sample(x, u, top_p=0.9), want[0]))
        with torch.cuda.stream(b):
            got.append((ais.top_logits(x, 50), want[1]))
    torch.cuda.synchronize()
    for g, w in got:
        assert all(torch.equal(p, q) for p, q in zip(g, w))


def test_an_ascending_row_and_a_descending_one():
    """Every entry beats those before it: the list of the largest overflows; and the other way round."""
    ais = _ais()
    V = 131072
    x = torch.stack([torch.arange(V), torch.arange(V).flip(0)]).float().cuda() * 1e-4
    for K in (1, 64, 1024):
        _check_top(x, K, 1.0, ais.top_logits(x, K))
    u = _u(2, 35)
    for how in (dict(top_k=100, top_p=0.9), dict(top_p=0.5), dict(top_k=3000), dict(min_p=0.2)):
        _check(x, u, *_sample(x, u, **how), **how)


# ------------------------------------------------------------------------------------------ top logits
def _check_top(x, K, tau, r):
    for i, row in enumerate(_np(x)):
        ids, values, lse = osel.top_row(row, K, tau)
        assert r.ids[i].tolist() == ids.tolist(), i
        assert np.array_equal(_np(r.values[i]), values)
        got = float(r.lse[i])
        assert (np.isnan(lse) and np.isnan(got)) or got == lse or abs(got - lse) <= HALF_STEP * abs(lse) + FULL


@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (33, 7), (1000, 1000), (4097, 1), (4097, 1024), (151936, 64), (262144, 300)])
def test_top_logits_sizes(V, K):
    ais = _ais()
    for dtype in DTYPES:
        for tau in (1.0, 0.3, 4.0):
            x = _logits(3, V, dtype, V + K, ld=V + 3, lead=1)
            _check_top(x, K, tau, ais.top_logits(x, K, temperature=tau))


def test_top_logits_of_equal_masked_and_bad_rows():
    ais = _ais()
    V, K = 40009, 100
    rng = np.random.default_rng(20)
    x = torch.from_numpy(rng.integers(0, 3, (8, V)) / 2.0).float().cuda()
    x[1] = 0.25
    x[2] = -np.inf
    x[2, [5, 9, 40000]] = torch.tensor([1.0, -2.0, 1.0], device="cuda")
    x[3] = -np.inf
    x[4, 3] = float("nan")
    x[5] *= 1e30
    x[6, ::2] = torch.finfo(torch.float32).min
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _check_top(x, K, 1.0, ais.top_logits(x, K, status=status))
    assert int(status.item()) == ais.FLAG_EMPTY | ais.FLAG_NONFINITE
    mask = torch.ones(8, dtype=torch.uint8, device="cuda")
    mask[7] = 0
    out = ais.TopLogits(torch.full((8, 128), 5, dtype=torch.int32, device="cuda")[:, :K], torch.full((8, 128), 5.0, device="cuda")[:, :K],
                        torch.empty(8, device="cuda"))
    ais.top_logits(x, K, mask=mask, out=out)
    assert (out.ids[7] == -1).all() and (out.values[7] == -np.inf).all() and float(out.lse[7]) == 0.0
    assert (out.ids._base[:, K:] == 5).all() and (out.values._base[:, K:] == 5.0).all()
    _check_top(x[:7], K, 1.0, ais.TopLogits(*(t[:7] for t in out)))


def test_longest_row():
    ais = _ais()
    x, u = _logits(2, ais.LOGITS_MAX_V, "fp32", 21), _u(2, 22)
    _check_top(x, 33, 1.0, ais.top_logits(x, 33))
    for how in (dict(top_p=0.9), dict(), dict(top_k=4000, min_p=0.001)):
        _check(x, u, *_sample(x, u, **how), **how)
