"""LayerNorm and its VJP (fpo_layernorm, fpo_layernorm_vjp) against their definitions in 64
bits, against differences, and at the sizes where the kernels change form.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp32 by 2^-24.
The fp32 arithmetic in front of it: a row sum of d terms in blocks of at most 16 per thread
and two short trees adds at most 40 roundings of 2^-24 relative to the sum of magnitudes, as
does the variance; what is subtracted around the mean is at most a few times the spread here,
so every element is held to 2^-24 * 400 of the row's largest plus the output rounding."""
import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
ARITH = 400 * 2.0 ** -24

# one element, one warp's rows, ragged rows of each form, its limits, and long rows
SHAPES = [("bf16", 1, 8), ("bf16", 7, 256), ("bf16", 200, 256), ("bf16", 33, 264),
          ("bf16", 19, 520), ("bf16", 5, 1032), ("bf16", 700, 2048), ("bf16", 3, 4096),
          ("bf16", 650, 4104), ("bf16", 1100, 4096), ("bf16", 2049, 1288), ("bf16", 1024, 2056),
          ("bf16", 4100, 2568), ("bf16", 4, 8192), ("bf16", 300, 8192), ("bf16", 70, 8200), ("bf16", 3, 20000),
          ("f32", 1, 1), ("f32", 9, 3), ("f32", 77, 33), ("f32", 130, 128), ("f32", 11, 260),
          ("f32", 300, 1023), ("f32", 1025, 4096), ("f32", 1111, 1028), ("f32", 3000, 520),
          ("f32", 5, 2047), ("f32", 6, 2052), ("f32", 3, 4099),
          ("f32", 2, 8191), ("f32", 3, 8192), ("f32", 400, 8192), ("f32", 256, 5004), ("f32", 4096, 2052),
          ("f32", 4096, 5000), ("f32", 70, 8193), ("f32", 3, 12000)]


def inputs(dtype, T, d, seed=0):
    g = torch.Generator().manual_seed(1000 * T + d + seed)
    x = torch.randn(T, d, generator=g) * torch.exp(0.7 * torch.randn(T, 1, generator=g))
    x += torch.randn(T, 1, generator=g)
    x[::5] *= 0.01  # rows whose spread is under the clamp
    gamma = 1 + 0.2 * torch.randn(d, generator=g)
    beta = 0.3 * torch.randn(d, generator=g)
    up = 1e-2 * torch.randn(T, d, generator=g)
    return [t.to(DT[dtype]).cuda() for t in (x, gamma, beta, up)]


def definition(x, gamma, beta, g, min_rms):
    x, gamma, beta, g = (t.double() for t in (x, gamma, beta, g))
    mu = x.mean(1, keepdim=True)
    sigma = ((x - mu) ** 2).mean(1, keepdim=True).add(EPS).sqrt()
    xh = (x - mu) / sigma
    u = gamma * g
    out = u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True)
    return dict(y=gamma * xh + beta, mean=mu[:, 0], rstd=1 / sigma[:, 0],
                g_out=out / sigma.clamp(min=min_rms), dgamma=(g * xh).sum(0), dbeta=g.sum(0),
                sgamma=(g * xh).abs().sum(0), sbeta=g.abs().sum(0))


def close(got, want, half, floor):
    got, want = got.double(), want.double()
    lim = half * want.abs() + (ARITH + half * ARITH) * floor + 1e-30
    bad = (got - want).abs() > lim
    assert not bad.any(), ((got - want).abs() / lim).max().item()


@pytest.mark.parametrize("dtype,T,d", SHAPES)
def test_forward_matches_the_definition(fpo, dtype, T, d):
    x, gamma, beta, g = inputs(dtype, T, d)
    ref = definition(x, gamma, beta, g, 0.5)
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.empty(T, device="cuda") for _ in range(2))
    fpo.layernorm(x, gamma, beta, y, eps=EPS, mean_out=mean, rstd_out=rstd)
    big = ref["y"].abs().amax(1, keepdim=True)
    # the mean's own error, relative to the row's spread
    off = 1 + x.double().abs().amax(1, keepdim=True) * ref["rstd"][:, None]
    close(y, ref["y"], HALF[dtype], (big + gamma.double().abs().max()) * off)
    close(mean, ref["mean"], 2.0 ** -24, x.double().abs().amax(1))
    close(rstd, ref["rstd"], 2.0 ** -24, ref["rstd"] * off[:, 0])
    # without a weight and a bias, and without the statistics
    fpo.layernorm(x, None, None, y, eps=EPS)
    plain = definition(x, torch.ones_like(gamma), torch.zeros_like(beta), g, 0.5)["y"]
    close(y, plain, HALF[dtype], (plain.abs().amax(1, keepdim=True) + 1) * off)


@pytest.mark.parametrize("min_rms", [0.0, 0.5])
@pytest.mark.parametrize("dtype,T,d", SHAPES)
def test_backward_matches_the_definition(fpo, dtype, T, d, min_rms):
    x, gamma, beta, g = inputs(dtype, T, d)
    ref = definition(x, gamma, beta, g, min_rms)
    out = torch.full_like(x, float("nan"))
    dg, db = (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
    fpo.layernorm_vjp(g, x, gamma, out, eps=EPS, min_rms=min_rms, dgamma=dg, dbeta=db)
    sigma = 1 / ref["rstd"][:, None]
    pref = 1 / sigma.clamp(min=min_rms)
    xh = (x.double() - ref["mean"][:, None]) / sigma
    off = 1 + x.double().abs().amax(1, keepdim=True) / sigma
    u = (gamma.double() * g.double()).abs().amax(1, keepdim=True)
    floor = u * pref * (1 + xh.abs().amax(1, keepdim=True)) * off
    close(out, ref["g_out"], HALF[dtype], floor)
    # sums of T terms, each xhat with the row's own error
    scale = (g.double() * (xh.abs() + 1) * off).abs().sum(0)
    close(dg, ref["dgamma"], 2.0 ** -24, scale)
    close(db, ref["dbeta"], 2.0 ** -24, ref["sbeta"])
    # each output alone, with the same bits
    out2 = torch.empty_like(out)
    fpo.layernorm_vjp(g, x, gamma, out2, eps=EPS, min_rms=min_rms)
    assert torch.equal(out, out2)
    dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
    fpo.layernorm_vjp(g, x, gamma, None, eps=EPS, min_rms=min_rms, dgamma=dg2)
    fpo.layernorm_vjp(g, x, gamma, None, eps=EPS, min_rms=min_rms, dbeta=db2)
    assert torch.equal(dg, dg2) and torch.equal(db, db2)


@pytest.mark.parametrize("dtype,d", [("f32", 33), ("f32", 512), ("f32", 2047), ("bf16", 64),
                                     ("bf16", 2048), ("bf16", 4096)])
def test_weight_sums_of_short_batches(fpo, dtype, d):
    """Batches on both sides of the largest that one cluster takes (no workspace), a block's rows
    and one more: dgamma and dbeta as the definition's, either one alone the same bits."""
    limit = 1
    while fpo.layernorm_vjp_workspace(limit + 1, d, 1 if dtype == "bf16" else 0) == 0:
        limit += 1
    assert limit >= 32
    for T in (1, 2, 9, limit - 1, limit, limit + 1):
        x, gamma, beta, g = inputs(dtype, T, d, seed=T)
        ref = definition(x, gamma, beta, g, 0.5)
        dg, db = (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
        out = torch.empty_like(x)
        fpo.layernorm_vjp(g, x, gamma, out, eps=EPS, dgamma=dg, dbeta=db)
        sigma = 1 / ref["rstd"][:, None]
        xh = (x.double() - ref["mean"][:, None]) / sigma
        off = 1 + x.double().abs().amax(1, keepdim=True) / sigma
        close(dg, ref["dgamma"], 2.0 ** -24, (g.double() * (xh.abs() + 1) * off).abs().sum(0))
        close(db, ref["dbeta"], 2.0 ** -24, ref["sbeta"])
        dg1, db1, out1 = torch.empty_like(dg), torch.empty_like(db), torch.empty_like(x)
        fpo.layernorm_vjp(g, x, gamma, out1, eps=EPS, dgamma=dg1)
        fpo.layernorm_vjp(g, x, gamma, None, eps=EPS, dbeta=db1)
        assert torch.equal(dg, dg1) and torch.equal(db, db1) and torch.equal(out, out1)


@pytest.mark.parametrize("case", ["first", "last", "mean"])
@pytest.mark.parametrize("dtype,T,d", [("bf16", 4100, 2568), ("f32", 4096, 5000), ("f32", 40, 5000)])
def test_outliers_and_large_means(fpo, dtype, T, d, case):
    """A feature 300 times the others (among the first elements, which the one-pass statistics
    take their origin from, or behind them), and a mean of 100 times the spread."""
    x, gamma, beta, g = inputs(dtype, T, d)
    x = x.clone()
    if case == "mean":
        x += 100 * x.float().std(1, keepdim=True).to(x.dtype)
    else:
        x[:, 3 if case == "first" else -2] *= 300
    ref = definition(x, gamma, beta, g, 0.0)
    y, out = torch.empty_like(x), torch.empty_like(x)
    dg, db = (torch.empty(d, device="cuda") for _ in range(2))
    fpo.layernorm(x, gamma, beta, y, eps=EPS)
    fpo.layernorm_vjp(g, x, gamma, out, eps=EPS, min_rms=0.0, dgamma=dg, dbeta=db)
    off = 1 + x.double().abs().amax(1, keepdim=True) * ref["rstd"][:, None]
    xh = (x.double() - ref["mean"][:, None]) * ref["rstd"][:, None]
    close(y, ref["y"], HALF[dtype], (ref["y"].abs().amax(1, keepdim=True) + gamma.double().abs().max()) * off)
    u = (gamma.double() * g.double()).abs().amax(1, keepdim=True)
    close(out, ref["g_out"], HALF[dtype],
          u * ref["rstd"][:, None] * (1 + xh.abs().amax(1, keepdim=True)) * off)
    close(dg, ref["dgamma"], 2.0 ** -24, (g.double() * (xh.abs() + 1) * off).abs().sum(0))
    close(db, ref["dbeta"], 2.0 ** -24, ref["sbeta"])


@pytest.mark.parametrize("dtype,T,d", [("bf16", 9, 264), ("bf16", 300, 2568), ("bf16", 4100, 2568),
                                       ("f32", 700, 33), ("f32", 4097, 2052), ("f32", 7, 9000)])
def test_nan_and_infinity_stay_in_their_row(fpo, dtype, T, d):
    """A row of x with a NaN or an infinity gives NaN throughout, one of g with a NaN too; the
    other rows are as without it (every form of the kernels)."""
    x, gamma, beta, g = inputs(dtype, T, d)
    y0, o0 = torch.empty_like(x), torch.empty_like(x)
    fpo.layernorm(x, gamma, beta, y0, eps=EPS)
    fpo.layernorm_vjp(g, x, gamma, o0, eps=EPS)
    bad, badg = x.clone(), g.clone()
    bad[0, d // 2] = float("nan")
    bad[T // 2, d - 1] = float("inf")
    badg[T - 1, 0] = float("nan")
    y, out = torch.empty_like(x), torch.empty_like(x)
    rstd = torch.empty(T, device="cuda")
    fpo.layernorm(bad, gamma, beta, y, eps=EPS, rstd_out=rstd)
    dg, db = (torch.zeros(d, device="cuda") for _ in range(2))
    fpo.layernorm_vjp(badg, bad, gamma, out, eps=EPS, dgamma=dg, dbeta=db)
    for r in (0, T // 2):
        assert y[r].isnan().all() and out[r].isnan().all() and rstd[r].isnan()
    assert out[T - 1].isnan().all() and dg.isnan().all() and db[0].isnan() and not db[1:].isnan().any()
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[0, T // 2]] = False
    assert torch.equal(y[keep], y0[keep])
    keep[T - 1] = False
    assert torch.equal(out[keep], o0[keep])


def test_calls_on_two_streams_at_once(fpo):
    """The stream kernels and the short-batch cluster, side by side on two streams."""
    sets = [inputs("bf16", T, 2568, seed=T) for T in (4100, 4100, 30)]
    def bufs(x):
        return [torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[1], device="cuda"),
                torch.empty(x.shape[1], device="cuda")]

    def call(s, b, stream):
        x, gamma, beta, g = s
        fpo.layernorm(x, gamma, beta, b[0], eps=EPS, stream=stream)
        fpo.layernorm_vjp(g, x, gamma, b[1], eps=EPS, dgamma=b[2], dbeta=b[3], workspace=b[4],
                          stream=stream)

    want = []
    for s in sets:
        b = bufs(s[0])
        b.append(torch.empty(max(256, fpo.layernorm_vjp_workspace(*s[0].shape)), dtype=torch.uint8,
                             device="cuda"))
        call(s, b, None)
        want.append(b)
    torch.cuda.synchronize()
    got = [[torch.empty_like(t) for t in b] for b in want]
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(10):
        for s, b, st in zip(sets, got, streams):
            call(s, b, st)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a[:4], b[:4]))


def test_a_wait_that_runs_out_leaves_nan(fpo):
    """With the wait limit at a microsecond the stream kernels may give up: every element is right
    or NaN; with the default limit the results are as before."""
    x, gamma, beta, g = inputs("bf16", 4100, 2568)
    d = x.shape[1]

    def call():
        y, out = torch.empty_like(x), torch.empty_like(x)
        dg, db = (torch.empty(d, device="cuda") for _ in range(2))
        fpo.layernorm(x, gamma, beta, y, eps=EPS)
        fpo.layernorm_vjp(g, x, gamma, out, eps=EPS, dgamma=dg, dbeta=db)
        torch.cuda.synchronize()
        return y, out, dg, db

    want = call()
    try:
        fpo.set_wait_limit_ns(1000)
        short = call()
    finally:
        fpo.set_wait_limit_ns(2_000_000_000)
    for a, b in zip(want, short):
        assert (b.isnan() | (a == b)).all()
    assert all(torch.equal(a, b) for a, b in zip(want, call()))


@pytest.mark.parametrize("T,d", [(3, 7), (4, 96)])
def test_backward_matches_differences(fpo, T, d):
    """g_out, dgamma and dbeta are the derivatives of <g, layernorm(x)>: fourth-order central
    differences of the 64-bit forward (step 1e-3: truncation and rounding under 1e-9 here)."""
    x, gamma, beta, g = inputs("f32", T, d, seed=3)
    x = x / x.std(1, keepdim=True)
    out, dg, db = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    fpo.layernorm_vjp(g, x, gamma, out, eps=EPS, min_rms=0.0, dgamma=dg, dbeta=db)
    x, gamma, beta, g = (t.double().cpu() for t in (x, gamma, beta, g))

    def f(xx, w, b):
        mu = xx.mean(1, keepdim=True)
        s = ((xx - mu) ** 2).mean(1, keepdim=True).add(EPS).sqrt()
        return float((g * ((xx - mu) / s * w + b)).sum())

    def diff(args, k):
        base, res, h = args[k], torch.empty_like(args[k]), 1e-3
        for i in range(base.numel()):
            v = []
            for c in (-2, -1, 1, 2):
                p = base.clone()
                p.view(-1)[i] += c * h
                v.append(f(*[p if j == k else a for j, a in enumerate(args)]))
            res.view(-1)[i] = (v[0] - 8 * v[1] + 8 * v[2] - v[3]) / (12 * h)
        return res

    args = (x, gamma, beta)
    for got, k in ((out, 0), (dg, 1), (db, 2)):
        want = diff(args, k)
        assert (got.double().cpu() - want).abs().max() < 1e-5 * want.abs().max() + 1e-7


def test_rows_do_not_touch_each_other_or_what_lies_behind(fpo):
    """Outputs end where the tensor ends; a NaN row stays in its row (and in the weight sums)."""
    for dtype, T, d in (("bf16", 9, 264), ("f32", 9, 33), ("bf16", 5, 4104), ("f32", 3, 8200)):
        x, gamma, beta, g = inputs(dtype, T, d)
        x[2, d // 2] = float("nan")
        y = torch.full((T + 2, d), 7.0, dtype=DT[dtype], device="cuda")
        o = torch.full((T + 2, d), 7.0, dtype=DT[dtype], device="cuda")
        fpo.layernorm(x, gamma, beta, y[:T], eps=EPS)
        fpo.layernorm_vjp(g, x, gamma, o[:T], eps=EPS)
        for t in (y, o):
            assert (t[T:] == 7.0).all()
            assert torch.isnan(t[2]).all()
            assert torch.isfinite(t[:2]).all() and torch.isfinite(t[3:T]).all()


def test_no_tokens_and_constant_rows(fpo):
    d = 64
    x = torch.empty(0, d, device="cuda")
    dg, db = torch.full((d,), 3.0, device="cuda"), torch.full((d,), 3.0, device="cuda")
    fpo.layernorm(x, None, None, torch.empty_like(x))
    fpo.layernorm_vjp(x, x, None, torch.empty_like(x), dgamma=dg, dbeta=db)
    assert (dg == 0).all() and (db == 0).all()
    # a constant row has sigma = sqrt(eps): y = beta exactly
    x = torch.full((3, d), 2.5, device="cuda")
    beta = torch.randn(d, device="cuda")
    y = torch.empty_like(x)
    fpo.layernorm(x, torch.randn(d, device="cuda"), beta, y, eps=EPS)
    assert torch.equal(y, beta.expand(3, d))


def test_large_offset_keeps_the_variance(fpo):
    """Rows at 1000 with a spread of 1: a variance from mean(x^2) - mean(x)^2 in fp32 would be
    off by about 6%; around the mean it keeps all but the input's own digits."""
    T, d = 64, 1024
    x = (1000 + torch.randn(T, d)).cuda()
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    fpo.layernorm(x, None, None, torch.empty_like(x), eps=EPS, mean_out=mean, rstd_out=rstd)
    want = 1 / (x.double().var(1, correction=0) + EPS).sqrt()
    assert ((rstd.double() - want) / want).abs().max() < 1e-5


@pytest.mark.parametrize("T, d", [(999, 1032), (60, 1032), (4099, 2200)])
def test_repeat_calls_other_streams_and_graphs(fpo, T, d):
    """Same bits from repeat calls, a side stream, two graphs that share a workspace (replayed
    one after the other), and replays on new inputs.  (60 rows: no workspace; 4099: the stream
    kernels.)"""
    x, gamma, beta, g = inputs("bf16", T, d)
    x2, _, _, g2 = inputs("bf16", T, d, seed=9)
    ws = torch.empty(fpo.layernorm_vjp_workspace(T, d), dtype=torch.uint8, device="cuda")

    def call(xx, gg, out, y, dg, db):
        fpo.layernorm(xx, gamma, beta, y, eps=EPS)
        fpo.layernorm_vjp(gg, xx, gamma, out, eps=EPS, dgamma=dg, dbeta=db, workspace=ws)

    def bufs():
        return [torch.zeros_like(x), torch.zeros_like(x)] + [torch.zeros(d, device="cuda")
                                                             for _ in range(2)]

    want, want2 = bufs(), bufs()
    call(x, g, *want)
    call(x2, g2, *want2)
    again = bufs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(x, g, *again)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    xs, gs = x.clone(), g.clone()
    graphs, outs = [], []
    for _ in range(2):
        o = bufs()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(xs, gs, *o)
        graphs.append(gr)
        outs.append(o)
    for gr in graphs:
        gr.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(want, o))
    xs.copy_(x2)
    gs.copy_(g2)
    for gr in graphs:
        gr.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(want2, o))


def test_signal_through_layernorm_feeds_the_update(fpo):
    """A target layer behind a LayerNorm: the error signal, composed through that norm's VJP,
    into the grouped update, as fpo_layer_signals composes it through an RMSNorm."""
    wl = synth.Workload("ln-chain", T=200, d=256, d_ff=384, V=1024, layers=2)
    inp = synth.make_all(wl)
    h, w, W_U, y = (inp[k].cuda() for k in ("h", "w", "W_U", "y"))
    gt = torch.empty_like(h)
    fpo.error_signal(h, w, W_U, y, gt)
    m = [synth.make_mlp_out(wl, l).cuda() for l in range(2)]
    gam = [synth.make_post_norm_w(wl, l).cuda() for l in range(2)]
    gs = [torch.empty_like(gt) for _ in range(2)]
    for l in range(2):
        fpo.layernorm_vjp(gt, m[l], gam[l], gs[l], eps=EPS, min_rms=0.5)
    A = [a.cuda() for a in inp["A"]]
    G = [torch.empty(wl.d, wl.d_ff, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    fpo.layer_update_grouped_signals(gs, A, 0.0, G_outs=G)
    for l in range(2):
        ref = definition(m[l], gam[l], torch.zeros_like(gam[l]), gt, 0.5)["g_out"]
        want = ref.t() @ A[l].double()
        # one bf16 rounding of the signal's elements and one of G's
        rel = (G[l].double() - want).norm() / want.norm()
        assert rel < 2 * 2.0 ** -8


def test_binding_refuses_wrong_tensors(fpo):
    x = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(16, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    for bad in (dict(gamma=w[:8]), dict(gamma=w.float()), dict(beta=w[:8]), dict(y=y[:3]),
                dict(y=y.float()), dict(mean_out=torch.empty(3, device="cuda"))):
        a = dict(gamma=w, beta=w, y=y) | bad
        with pytest.raises(ValueError):
            fpo.layernorm(x, a.pop("gamma"), a.pop("beta"), a.pop("y"), **a)
    with pytest.raises(ValueError):
        fpo.layernorm_vjp(x[:3], x, w, y)
    with pytest.raises(ValueError):
        fpo.layernorm_vjp(x, x, w, y, dgamma=torch.empty(16, device="cuda").bfloat16())
    with pytest.raises(ValueError):
        fpo.layernorm(x.t(), None, None, torch.empty_like(x.t()))  # not contiguous
    with pytest.raises(fpo.FpoError):
        fpo.layernorm(x, w, w, x)
    with pytest.raises(fpo.FpoError):
        fpo.layernorm_vjp(x, x, w, x)
    assert np.isfinite(EPS)
