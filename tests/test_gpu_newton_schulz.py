"""Newton-Schulz orthogonalisation and the Muon step (fpo_orthogonalize_grouped,
fpo_layer_muon_grouped) against their definitions in 64 bits.

Tolerances, as the 2-norm of the difference over that of the result.
bf16: the operands X, A, B of each product are rounded to fp16, at random within 2^-12 of their
value (rms 2^-12 / sqrt 3 = 1.4e-4 each).  A perturbation of X_k reaches the result times at
most p' of the steps behind it where the linear term does not carry it; over the five steps
of the quintic these add up to at most 14 times 1.4e-4 = 2e-3 (an emulation of the roundings in
64 bits gives 0.4e-3 to 1.9e-3 for sides 64 to 768, ranks from 1 up).  The output's own rounding
to bf16 adds 2^-8 / sqrt 3 = 2.3e-3 at most.  Limit 4.5e-3.
fp32: operands of two fp16 numbers are within 2^-24; every element of a product is a sum of
64-deep parts, each truncated in its last 4 or 5 additions (2^-23 of the part, half of it on
average), added with one rounding each.  2e-3 * (2^-24 + 2^-23) / 2^-12 = 1.5e-6 for the
operands, and with A's error (5 * 2^-24 on average) through b and c like X's: 14 * 5 * 2^-24
= 4e-6; limit 1e-5.  A matrix of low rank has directions in which X is nothing: errors there
grow by a = 3.44 a step.  X's own rounding to fp32, 480 * 2^-24 = 3e-5 of the largest singular
value, and what the error of B = b A + .. leaves there in the first step, |b| 5 * 2^-24 * 3.44^4
= 4.78 * 3e-7 * 140 = 2e-4 if all of it points there; limit 2e-4."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
QUINTIC = (3.4445, -4.7750, 2.0315)


def f32(v):
    return torch.tensor(v, dtype=torch.float32).double().item()


def definition(G, steps=5, coeffs=None, eps=1e-7):
    X = G.double()
    X = X / max(X.norm().item(), eps)
    tall = X.shape[0] > X.shape[1]
    X = X.mT if tall else X
    for k in range(steps):
        a, b, c = (f32(v) for v in (QUINTIC if coeffs is None else coeffs[k]))
        A = X @ X.mT
        X = a * X + (b * A + c * A @ A) @ X
    return X.mT if tall else X


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def matrix(rows, cols, kind, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + cols)

    def n(*s):
        return torch.randn(*s, generator=gen, device="cuda")

    if kind == "full":
        return n(rows, cols)
    if kind.startswith("rank"):
        r = int(kind[4:])
        return 1e-6 * n(rows, r) @ n(r, cols)
    # singular values over four decades
    m = min(rows, cols)
    U, V = torch.linalg.qr(n(rows, m))[0], torch.linalg.qr(n(cols, m))[0]
    return (U * torch.logspace(2, -2, m, device="cuda")) @ V.mT


SHAPES16 = [(8, 8), (16, 264), (64, 64), (256, 384), (384, 256), (264, 520), (520, 264),
            (1024, 256), (776, 1544), (1544, 776), (8, 2048)]
SHAPES32 = [(1, 1), (1, 7), (9, 1), (33, 70), (64, 64), (70, 33), (255, 257), (300, 517),
            (517, 300), (767, 1025), (700, 2049), (2049, 700)]


def limit(dtype, kind):
    if dtype == "bf16":
        return 4.5e-3
    return 1e-5 if kind == "full" else 2e-4


@pytest.mark.parametrize("kind", ["full", "rank1", "rank5", "decades"])
@pytest.mark.parametrize("dtype,rows,cols", [("bf16", *s) for s in SHAPES16] +
                         [("f32", *s) for s in SHAPES32])
def test_orthogonalize_matches_the_definition(fpo, dtype, rows, cols, kind):
    Gs = [matrix(rows, cols, kind, seed=l).to(DT[dtype]) for l in range(3)]
    Os = [torch.full_like(G, float("nan")) for G in Gs]
    ws = fpo.orthogonalize_grouped(Gs, Os)
    assert fpo.get_device_status(ws) == fpo.OK
    for G, O in zip(Gs, Os):
        assert rel(O, definition(G)) < limit(dtype, kind)


@pytest.mark.parametrize("rows,cols", [(8, 8), (64, 256), (2048, 32), (16, 8192)])
def test_small_sides_are_exact_to_the_rounding(fpo, rows, cols):
    """bf16 matrices with a side of at most 64: the fp32 products' 1e-5, and the rounding of the
    result, 2^-8 of every element at most, 2^-8 / sqrt 3 in norm where they are spread."""
    Gs = [matrix(rows, cols, "full", seed=l).bfloat16() for l in range(3)]
    Os = [torch.empty_like(G) for G in Gs]
    fpo.orthogonalize_grouped(Gs, Os)
    for G, O in zip(Gs, Os):
        want = definition(G)
        assert ((O.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * want.norm()).all()
        assert rel(O, want.bfloat16().double()) < 1e-3  # few round the other way


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_result_is_near_orthogonal(fpo, dtype):
    """Singular values of a square Gaussian matrix's bulk land in the quintic's band."""
    G = matrix(512, 1024, "full").to(DT[dtype])
    O = torch.empty_like(G)
    fpo.orthogonalize_grouped([G], [O])
    s = torch.linalg.svdvals(O.double())
    assert s.min() > 0.65 and s.max() < 1.25


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_other_coefficients_and_step_counts(fpo, dtype):
    """A schedule of its own per step, the cubic (1.5, -0.5, 0), one step, ten steps."""
    G = matrix(200, 328, "full").to(DT[dtype])
    schedules = [[(1.5, -0.5, 0.0)] * 10, [(2.0, -1.5, 0.5)] * 3,
                 [(3.9, -8.6, 4.9), (3.4445, -4.775, 2.0315), (1.875, -1.25, 0.375)],
                 [(1.0, 0.0, 0.0)], [(3.4445, -4.775, 2.0315)]]
    for co in schedules:
        O = torch.empty_like(G)
        ws = fpo.orthogonalize_grouped([G], [O], steps=len(co), coeffs=co)
        assert fpo.get_device_status(ws) == fpo.OK
        # as the module's limits: the errors of ten steps add up to at most twice those of five
        assert rel(O, definition(G, len(co), co)) < 2 * limit(dtype, "full")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_zero_matrices_and_the_norm_floor(fpo, dtype):
    """The result does not depend on G's scale (powers of two: the same bits) down to where
    squares leave fp32's range; a zero matrix gives zeros; below eps the norm is eps."""
    G = matrix(72, 136, "full").to(DT[dtype])
    ref = torch.empty_like(G)
    fpo.orthogonalize_grouped([G], [ref], eps=1e-30)
    for e in (-60, 40, 80):
        O = torch.empty_like(G)
        fpo.orthogonalize_grouped([G * 2.0 ** e], [O], eps=1e-30)
        assert rel(O, ref.double()) < 1e-2 if dtype == "bf16" else torch.equal(O, ref) or \
            rel(O, ref.double()) < 1e-5
    O = torch.full_like(G, 3.0)
    fpo.orthogonalize_grouped([torch.zeros_like(G)], [O])
    assert (O == 0).all()
    small = G * 2.0 ** -40  # norm 9e-11
    fpo.orthogonalize_grouped([small], [O], eps=1e-7)
    want = definition(small, eps=f32(1e-7))
    assert rel(O, want) < limit(dtype, "full")


def test_a_bad_matrix_spoils_itself_only(fpo):
    for dtype in ("bf16", "f32"):
        Gs = [matrix(72, 136, "full", seed=l).to(DT[dtype]) for l in range(3)]
        ref = [torch.empty_like(G) for G in Gs]
        fpo.orthogonalize_grouped(Gs, ref)
        for v in (float("nan"), float("inf")):
            bad = [G.clone() for G in Gs]
            bad[1][5, 7] = v
            Os = [torch.zeros_like(G) for G in Gs]
            ws = fpo.orthogonalize_grouped(bad, Os)
            assert fpo.get_device_status(ws) == fpo.OK
            assert torch.isnan(Os[1]).all()
            assert torch.equal(Os[0], ref[0]) and torch.equal(Os[2], ref[2])


# (bf16 512 x 2048: one launch for one matrix, a launch per product and wider tiles for four;
# f32: with and without k-blocks in ranges; 700 x 2049: 128-column tiles for one, 256 for four)
@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 264, 520), ("bf16", 512, 2048),
                                             ("bf16", 2048, 520), ("f32", 129, 263),
                                             ("f32", 257, 2300), ("f32", 2300, 130),
                                             ("f32", 3, 5000), ("f32", 700, 2049),
                                             ("f32", 2049, 700)])
def test_in_place_groups_streams_and_graphs(fpo, dtype, rows, cols):
    """In place, in any group, on another stream, and in two graphs that share a workspace:
    the same bits.  Nothing behind the outputs is written."""
    Gs = [matrix(rows, cols, "full", seed=l).to(DT[dtype]) for l in range(4)]
    ref = [torch.empty_like(G) for G in Gs]
    fpo.orthogonalize_grouped(Gs, ref)
    alone = torch.empty_like(Gs[2])
    fpo.orthogonalize_grouped([Gs[2]], [alone])
    assert torch.equal(alone, ref[2])
    inpl = [G.clone() for G in Gs]
    fpo.orthogonalize_grouped(inpl, inpl)
    assert all(torch.equal(a, b) for a, b in zip(inpl, ref))
    swap = [G.clone() for G in Gs[:2]]
    fpo.orthogonalize_grouped(swap, swap[::-1])  # O[0] is G[1] and the other way around
    assert torch.equal(swap[1], ref[0]) and torch.equal(swap[0], ref[1])
    guard = torch.full((rows + 2, cols), 5.0, dtype=DT[dtype], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    fpo.orthogonalize_grouped([Gs[0]], [guard[:rows]], stream=s)
    s.synchronize()
    assert torch.equal(guard[:rows], ref[0]) and (guard[rows:] == 5.0).all()
    dt = fpo.BF16 if dtype == "bf16" else fpo.F32
    ws = torch.empty(fpo.orthogonalize_workspace(2, rows, cols, dt), dtype=torch.uint8,
                     device="cuda")
    src = [G.clone() for G in Gs[:2]]
    graphs, outs = [], []
    for _ in range(2):
        o = [torch.empty_like(G) for G in src]
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            fpo.orthogonalize_grouped(src, o, workspace=ws)
        graphs.append(gr)
        outs.append(o)
    for gr in graphs + graphs:
        gr.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], ref[0]) and torch.equal(o[1], ref[1])
    for t, G in zip(src, Gs[2:]):
        t.copy_(G)
    for gr in graphs:
        gr.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], ref[2]) and torch.equal(o[1], ref[3])


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 40, 24), ("f32", 33, 2100)])
def test_large_group(fpo, dtype, rows, cols):
    """64 layers, the most one call takes, and a workspace of exactly the queried size with
    guard bytes behind it."""
    n = 64
    Gs = [matrix(rows, cols, "full", seed=l).to(DT[dtype]) for l in range(n)]
    Os = [torch.empty_like(G) for G in Gs]
    need = fpo.orthogonalize_workspace(n, rows, cols, fpo.BF16 if dtype == "bf16" else fpo.F32)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    fpo.orthogonalize_grouped(Gs, Os, workspace=ws[:need])
    assert (ws[need:] == 171).all()
    for G, O in zip(Gs, Os):
        assert rel(O, definition(G)) < (4.5e-3 if dtype == "bf16" else 1e-5)


def test_calls_on_two_streams_at_once(fpo):
    """The one-launch form (every cluster of a call waits for the others) and the launches per
    product, calls overlapping on three streams with workspaces of their own."""
    shapes = [("bf16", 1024, 1024, 2), ("bf16", 512, 2048, 2), ("f32", 257, 2300, 2)]
    jobs = []
    for dtype, r, c, n in shapes:
        G = [matrix(r, c, "full", seed=l).to(DT[dtype]) for l in range(n)]
        ref = [torch.empty_like(t) for t in G]
        fpo.orthogonalize_grouped(G, ref)
        O = [torch.full_like(t, float("nan")) for t in G]
        need = fpo.orthogonalize_workspace(n, r, c, fpo.BF16 if dtype == "bf16" else fpo.F32)
        jobs.append((G, O, ref, torch.empty(need, dtype=torch.uint8, device="cuda"),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for G, O, _, ws, s in jobs:
            fpo.orthogonalize_grouped(G, O, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for _, O, ref, ws, _ in jobs:
        assert fpo.get_device_status(ws) == fpo.OK
        assert all(torch.equal(a, b) for a, b in zip(O, ref))


@pytest.mark.parametrize("dtype,rows,cols,n", [("bf16", 512, 2048, 1), ("bf16", 512, 2048, 8),
                                               ("f32", 257, 2300, 2), ("f32", 700, 2049, 4)])
def test_waits_that_run_out_are_reported(fpo, dtype, rows, cols, n):
    """Every form with a wait limit far below the first operands' way in: the status says so, and
    the next call, with the default limit and the same workspace, gives the same bits as before."""
    G = [matrix(rows, cols, "full", seed=l).to(DT[dtype]) for l in range(n)]
    ref, O = ([torch.empty_like(t) for t in G] for _ in range(2))
    ws = fpo.orthogonalize_grouped(G, ref)
    assert fpo.get_device_status(ws) == fpo.OK
    for _ in range(2):
        try:
            fpo.set_wait_limit_ns(100)
            fpo.orthogonalize_grouped(G, O, workspace=ws)
            assert fpo.get_device_status(ws) == 9  # FPO_ERR_TIMEOUT
        finally:
            fpo.set_wait_limit_ns(2_000_000_000)
    fpo.orthogonalize_grouped(G, O, workspace=ws)
    assert fpo.get_device_status(ws) == fpo.OK
    assert all(torch.equal(a, b) for a, b in zip(O, ref))


# ------------------------------------------------------------------------ Muon step
def muon_inputs(dtype, T, d, d_ff, n, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + T + 3 * d + d_ff)

    def r(*s):
        return torch.randn(*s, generator=gen, device="cuda")

    gs = [(1e-3 * r(T, d)).to(DT[dtype]) for _ in range(n)]
    As = [(torch.nn.functional.silu(r(T, d_ff)) * r(T, d_ff)).to(DT[dtype]) for _ in range(n)]
    W = [0.02 * r(d, d_ff) for _ in range(n)]
    M = [5e-4 * math.sqrt(max(T, 1)) * r(d, d_ff) for _ in range(n)]
    return gs, As, W, M


def muon_definition(g, A, W, M, lr, mu, wd, scale, nesterov):
    G = g.double().mT @ A.double()
    M = f32(mu) * M.double() + G
    U = G + f32(mu) * M if nesterov else M
    O = definition(U)
    return M, W.double() * f32(1 - f32(lr) * f32(wd)) - f32(lr) * f32(scale) * O, O


MUON = [("bf16", 200, 256, 384, 2), ("bf16", 1, 64, 136, 3), ("bf16", 700, 520, 264, 2),
        ("bf16", 4160, 64, 136, 2), ("bf16", 9000, 72, 64, 1), ("bf16", 4200, 1032, 2056, 2),
        ("bf16", 0, 64, 64, 1), ("f32", 128, 64, 256, 2), ("f32", 77, 65, 33, 2),
        ("f32", 0, 9, 30, 1), ("f32", 300, 31, 500, 1)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype,T,d,d_ff,n", MUON)
def test_muon_step_matches_the_definition(fpo, dtype, T, d, d_ff, n, nesterov):
    gs, As, W, M = muon_inputs(dtype, T, d, d_ff, n)
    lr, mu, wd, scale = 2e-2, 0.9, 0.1, 0.5
    want = [muon_definition(*t, lr, mu, wd, scale, nesterov) for t in zip(gs, As, W, M)]
    Wo = [torch.empty(d, d_ff, dtype=DT[dtype], device="cuda") for _ in range(n)]
    W0 = [w.clone() for w in W]
    opt = fpo.muon_desc(lr=lr, momentum=mu, weight_decay=wd, scale=scale, nesterov=nesterov)
    ws = fpo.layer_muon_grouped(gs, As, opt, W, M, W_outs=Wo)
    assert fpo.get_device_status(ws) == fpo.OK
    for l in range(n):
        Mr, Wr, Or = want[l]
        # sums of T products: tensor-core sums truncate, at most 2^-23 a 16-deep step of the
        # running sum's size; fp32 sums round
        assert rel(M[l], Mr) < (T / 16 + 2) * 2.0 ** -23 + 1e-6
        # the step alone, so that W's size does not hide it; the fp32 master rounds once or
        # twice, 2^-23 of W
        step = W[l].double() - W0[l].double() * f32(1 - f32(lr) * f32(wd))
        tol = 2.5e-3 if dtype == "bf16" else 2e-5
        floor = 2.0 ** -23 * W0[l].double().norm() / (lr * scale * Or.norm())
        assert rel(step, -f32(lr) * f32(scale) * Or) < tol + floor
        assert torch.equal(Wo[l], W[l].to(DT[dtype]))


def test_many_tokens_of_one_sign(fpo):
    """The tensor core's sums truncate, so those of positive products come out too small: by up to
    2^-23 of the running sum (on average half the final one) at each of the 256 16-deep steps of
    the 4096 tokens of one accumulator, and no more for more tokens."""
    T, d, d_ff = 16384, 64, 128
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = torch.rand(T, d, generator=gen, device="cuda").bfloat16()
    A = torch.rand(T, d_ff, generator=gen, device="cuda").bfloat16()
    W, M = (torch.zeros(d, d_ff, device="cuda") for _ in range(2))
    fpo.layer_muon_grouped([g], [A], fpo.muon_desc(lr=1e-3), [W], [M])
    assert rel(M, g.double().T @ A.double()) < 256 * 2.0 ** -24 + 8 * 2.0 ** -24


def test_muon_step_without_weight_copy_in_a_graph(fpo):
    """W_outs omitted; repeated entries of g and A; replays step the same buffers, bit for bit
    as eager calls do."""
    gs, As, W, M = muon_inputs("bf16", 96, 72, 136, 2)
    gs, As = [gs[0], gs[0]], [As[0], As[0]]
    W = [W[0], W[0].clone()]
    M = [M[0], M[0].clone()]
    W2, M2 = [w.clone() for w in W], [m.clone() for m in M]
    opt = fpo.muon_desc(lr=1e-2)
    for _ in range(3):
        fpo.layer_muon_grouped(gs, As, opt, W, M)
    assert torch.equal(W[0], W[1]) and torch.equal(M[0], M[1])
    ws = torch.empty(fpo.layer_muon_workspace(2, 72, 136), dtype=torch.uint8, device="cuda")
    fpo.layer_muon_grouped(gs, As, opt, [w.clone() for w in W2], [m.clone() for m in M2],
                           workspace=ws)
    gr = torch.cuda.CUDAGraph()
    keep = [t.clone() for t in W2 + M2]
    with torch.cuda.graph(gr):
        fpo.layer_muon_grouped(gs, As, opt, W2, M2, workspace=ws)
    for t, k in zip(W2 + M2, keep):
        assert torch.equal(t, k)
    for _ in range(3):
        gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(W[0], W2[0]) and torch.equal(M[1], M2[1])


def test_training_step_through_layernorm_and_muon(fpo):
    """The operators together: LayerNorm forward, the signal through its VJP, the Muon step
    of a down-projection and of a gate matrix (taller than wide)."""
    T, d, d_ff = 192, 136, 264
    gen = torch.Generator(device="cuda").manual_seed(5)

    def r(*s):
        return torch.randn(*s, generator=gen, device="cuda")

    x, up = r(T, d).bfloat16(), (1e-2 * r(T, d)).bfloat16()
    gamma, beta = (1 + 0.1 * r(d)).bfloat16(), (0.1 * r(d)).bfloat16()
    y, g = torch.empty_like(x), torch.empty_like(x)
    dgam, dbet = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    fpo.layernorm(x, gamma, beta, y)
    fpo.layernorm_vjp(up, x, gamma, g, min_rms=0.0, dgamma=dgam, dbeta=dbet)
    h = (torch.nn.functional.silu(r(T, d_ff)) * r(T, d_ff)).bfloat16()
    W3, M3 = 0.02 * r(d, d_ff), torch.zeros(d, d_ff, device="cuda")
    W1, M1 = 0.02 * r(d_ff, d), torch.zeros(d_ff, d, device="cuda")
    opt = fpo.muon_desc(lr=1e-2, scale=1.0)
    ref3 = muon_definition(g, h, W3, M3, 1e-2, 0.95, 0.0, 1.0, True)
    ref1 = muon_definition(h, y, W1, M1, 1e-2, 0.95, 0.0, 1.0, True)
    fpo.layer_muon_grouped([g], [h], opt, [W3], [M3])
    fpo.layer_muon_grouped([h], [y], opt, [W1], [M1])
    # x's gradient is that of autograd, in 64 bits
    xd = x.double().requires_grad_()
    (torch.nn.functional.layer_norm(xd, (d,), gamma.double(), beta.double(), 1e-5) *
     up.double()).sum().backward()
    assert rel(g, xd.grad) < 2.0 ** -8
    assert rel(W3, ref3[1]) < 2.5e-3 and rel(W1, ref1[1]) < 2.5e-3


def test_binding_refuses_wrong_tensors(fpo):
    G = torch.zeros(16, 24, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        fpo.orthogonalize_grouped([G, G[:8]], [G, G])
    with pytest.raises(ValueError):
        fpo.orthogonalize_grouped([G], [G.float()])
    with pytest.raises(ValueError):
        fpo.orthogonalize_grouped([G], [G, G])
    with pytest.raises(ValueError):
        fpo.orthogonalize_grouped([G], [G], steps=2, coeffs=[(1, 0, 0)])
    with pytest.raises(fpo.FpoError):
        fpo.orthogonalize_grouped([G], [G], steps=0)
    with pytest.raises(fpo.FpoError):
        fpo.orthogonalize_grouped([G], [G], steps=2, coeffs=[(1e4, 0, 0)] * 2)
    with pytest.raises(fpo.FpoError):  # a smaller workspace
        fpo.orthogonalize_grouped([G], [G], workspace=torch.empty(1024, dtype=torch.uint8,
                                                                  device="cuda"))
    gs, As, W, M = muon_inputs("bf16", 16, 16, 24, 1)
    opt = fpo.muon_desc()
    for bad in (dict(gs=[gs[0][:8]]), dict(W=[W[0].bfloat16()]), dict(M=[M[0][:8]]),
                dict(M=[]), dict(W_outs=[W[0]])):
        a = dict(gs=gs, As=As, W=W, M=M, W_outs=None) | bad
        with pytest.raises(ValueError):
            fpo.layer_muon_grouped(a["gs"], a["As"], opt, a["W"], a["M"], W_outs=a["W_outs"])
