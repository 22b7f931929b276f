"""The linear layer and its backward pass (fpo_linear, fpo_linear_vjp) against their definitions in
64 bits, against differences, and at the sizes where the kernels change form.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp32 by 2^-24.  The sums
in front of it: the tensor cores take 16 products at a time and add them to the fp32 sum, k / 16 + 32
additions with those of the parts of split tiles, each at most 2^-23 off relative to the sum of
magnitudes S (it may cut digits off); the fp32 kernels add at most k products in a row, 2^-24 each.
The activations' fp32 forms are within 2^-17 of the value (the exponential's argument has up to 7
bits in front of the point), and none has a slope above 1.13."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]

# one element; one to four tokens of wide layers; the padded token counts of short batches and their limits;
# a tile's edges; single CTAs' tiles of 64 and 128 columns; pair tiles of 128 columns; k ranges of few
# tiles; a split last wave; long and short k
SHAPES = [("bf16", 1, 8, 8), ("bf16", 1, 4096, 1416), ("bf16", 1, 72, 11008), ("bf16", 3, 64, 128),
          ("bf16", 2, 4104, 136), ("bf16", 4, 11008, 72),
          ("bf16", 5, 1032, 264), ("bf16", 16, 200, 136), ("bf16", 17, 264, 1000), ("bf16", 32, 4096, 1000),
          ("bf16", 33, 520, 72), ("bf16", 64, 1032, 640),
          ("bf16", 65, 2056, 264), ("bf16", 128, 1024, 2056), ("bf16", 64, 4096, 4104), ("bf16", 129, 64, 264), ("bf16", 200, 256, 384),
          ("bf16", 513, 1032, 4104), ("bf16", 1024, 11008, 1032),
          ("bf16", 256, 4096, 512), ("bf16", 257, 2056, 1032), ("bf16", 700, 4096, 512),
          ("bf16", 384, 4096, 4096), ("bf16", 1024, 8, 4104), ("bf16", 2000, 136, 8),
          ("bf16", 5000, 2056, 2048), ("bf16", 5000, 11008, 2048),
          ("bf16", 9000, 1024, 1288), ("f32", 1, 1, 1), ("f32", 7, 3, 5), ("f32", 1, 700, 1001),
          ("f32", 2, 4096, 72), ("f32", 3, 301, 1000), ("f32", 5, 1024, 264), ("f32", 11, 2049, 65),
          ("f32", 16, 2048, 136), ("f32", 17, 2048, 136),
          ("f32", 130, 67, 129), ("f32", 200, 256, 384), ("f32", 777, 767, 129), ("f32", 65, 2049, 64)]


def act_of(fpo, name):
    return {"none": fpo.ACT_NONE, "relu": fpo.ACT_RELU, "gelu": fpo.ACT_GELU,
            "gelu_tanh": fpo.ACT_GELU_TANH, "silu": fpo.ACT_SILU}[name]


def act64(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)  # 0 at 0 (clamp's autograd form would give 1 there)
    z = z.detach().clone().requires_grad_()
    act64(name, z).sum().backward()
    return z.grad


def inputs(dtype, T, k, n, seed=0):
    g = torch.Generator().manual_seed(T * 7919 + k * 31 + n + seed)
    r = lambda *s: torch.randn(*s, generator=g).to(DT[dtype]).cuda()  # noqa: E731
    return dict(x=r(T, k), W=(r(n, k) * (1.5 / math.sqrt(k))).to(DT[dtype]), bias=r(n), residual=r(T, n),
                dy=r(T, n), z=r(T, n), z_in=r(T, k))


def acc(dtype, k, magnitudes):
    """What the sums of k products may be off by."""
    steps = (k / 16 + 32) * 2.0 ** -23 if dtype == "bf16" else (k + 8) * 2.0 ** -24
    return steps * magnitudes


def close(got, want, half, floor):
    got, want = got.double(), want.double()
    assert not got.isnan().any()
    lim = half * want.abs() + (1 + half) * floor + 1e-30
    off = ((got - want).abs() / lim).max().item()
    assert off <= 1, off


@pytest.mark.parametrize("dtype,T,k,n", SHAPES)
def test_forward_matches_the_definition(fpo, dtype, T, k, n):
    d = inputs(dtype, T, k, n)
    z0 = d["x"].double() @ d["W"].double().t()
    floor = acc(dtype, k, d["x"].double().abs() @ d["W"].double().abs().t())
    for i, act in enumerate(ACTS):
        for bias, res, keep in ((True, True, True), (False, i % 2 == 0, i % 2 == 1)):
            buf = torch.full((T + 3, n), 7.0, dtype=DT[dtype], device="cuda")
            zbuf = torch.full((T + 3, n), 7.0, dtype=DT[dtype], device="cuda")
            ws = fpo.linear(d["x"], d["W"], buf[:T], bias=d["bias"] if bias else None, act=act_of(fpo, act),
                            residual=d["residual"] if res else None, z_out=zbuf[:T] if keep else None)
            assert fpo.get_device_status(ws) == fpo.OK
            z = z0 + d["bias"].double() if bias else z0
            f = floor + 2.0 ** -23 * (z.abs() + z0.abs())
            y = act64(act, z)
            fy = 1.13 * f + 2.0 ** -17 * y.abs()
            if res:
                y = y + d["residual"].double()
                fy = fy + 2.0 ** -23 * y.abs()
            close(buf[:T], y, HALF[dtype], fy)
            if keep:
                close(zbuf[:T], z, HALF[dtype], f)
            # rows behind the batch stay as they were
            assert (buf[T:] == 7).all() and (zbuf[T:] == 7).all() and (keep or (zbuf == 7).all())


@pytest.mark.parametrize("dtype,T,k,n", SHAPES)
def test_backward_matches_the_definition(fpo, dtype, T, k, n):
    d = inputs(dtype, T, k, n)
    half = HALF[dtype]
    cases = [("none", "none"), ("none", "gelu_tanh"), ("silu", "none"), ("gelu", "relu"),
             ("relu", "gelu"), ("gelu_tanh", "silu")]
    for act, act_in in cases:
        dx = torch.full((T + 2, k), 7.0, dtype=DT[dtype], device="cuda")
        dW = torch.full((n, k), 7.0, dtype=DT[dtype], device="cuda")
        db = torch.full((n,), 7.0, device="cuda")
        ws = fpo.linear_vjp(d["dy"], d["x"], d["W"], dx[:T], act=act_of(fpo, act),
                            z=d["z"] if act != "none" else None, act_in=act_of(fpo, act_in),
                            z_in=d["z_in"] if act_in != "none" else None, dW=dW, dbias=db)
        assert fpo.get_device_status(ws) == fpo.OK
        s, s_in = slope64(act, d["z"].double()), slope64(act_in, d["z_in"].double())
        dz = d["dy"].double() * s
        # the slopes' own error, on values of at most about 1, and dZ's rounding in the products
        edz = d["dy"].double().abs() * 2.0 ** -17 if act != "none" else torch.zeros_like(dz)
        rdz = edz + (half * dz.abs() if act != "none" else 0)
        W, x = d["W"].double(), d["x"].double()
        v = dz @ W
        fv = acc(dtype, n, dz.abs() @ W.abs()) + 1.01 * rdz @ W.abs()
        close(dx[:T], v * s_in, half, 1.13 * fv + 2.0 ** -17 * v.abs() * (act_in != "none"))
        close(dW, dz.t() @ x, half, acc(dtype, T, dz.t().abs() @ x.abs()) + 1.01 * rdz.t() @ x.abs())
        # a thread's rows, the block's 16, the ranges
        close(db, dz.sum(0), 2.0 ** -24, (T / 16 + 640) * 2.0 ** -24 * dz.abs().sum(0) + edz.sum(0))
        assert (dx[T:] == 7).all()


@pytest.mark.parametrize("dtype,T,k,n", [("bf16", 200, 256, 384), ("bf16", 5, 72, 136), ("f32", 33, 70, 65)])
def test_outputs_alone(fpo, dtype, T, k, n):
    d = inputs(dtype, T, k, n)
    silu = fpo.ACT_SILU

    def run(dx=False, dW=False, db=False):
        out = (torch.empty(T, k, dtype=DT[dtype], device="cuda") if dx else None,
               torch.empty(n, k, dtype=DT[dtype], device="cuda") if dW else None,
               torch.empty(n, device="cuda") if db else None)
        fpo.linear_vjp(d["dy"], d["x"] if dW else None, d["W"] if dx else None, out[0], act=silu, z=d["z"],
                       act_in=silu if dx else 0, z_in=d["z_in"] if dx else None, dW=out[1], dbias=out[2])
        return out

    whole = run(True, True, True)
    for i in range(3):
        one = run(*[j == i for j in range(3)])
        assert torch.equal(one[i], whole[i])


# one range of rows, a cluster's and, above 2048 (with an activation) and 8192 rows, joined by counters;
# column groups that end inside; more column groups than blocks are wanted
@pytest.mark.parametrize("dtype,T,n", [("bf16", 1, 8), ("bf16", 64, 136), ("bf16", 65, 136), ("bf16", 257, 264),
                                       ("bf16", 513, 20000), ("bf16", 2048, 136), ("bf16", 2049, 1032),
                                       ("bf16", 8192, 72), ("bf16", 8193, 72), ("f32", 63, 7), ("f32", 129, 260),
                                       ("f32", 513, 1025), ("f32", 300, 40004), ("f32", 2049, 33), ("f32", 8193, 20)])
def test_bias_sums(fpo, dtype, T, n):
    d = inputs(dtype, T, 1 if dtype == "f32" else 8, n)
    for act in ("none", "silu"):
        db = torch.full((n + 4,), 7.0, device="cuda")
        z = d["z"] if act != "none" else None
        for _ in range(2):
            ws = fpo.linear_vjp(d["dy"], None, None, None, act=act_of(fpo, act), z=z, dbias=db[:n])
            assert fpo.get_device_status(ws) == fpo.OK
            dz = d["dy"].double() * slope64(act, d["z"].double())
            edz = d["dy"].double().abs() * 2.0 ** -17 if act != "none" else torch.zeros_like(dz)
            # a thread's rows, the block's 16, the ranges
            close(db[:n], dz.sum(0), 2.0 ** -24, (T / 16 + 640) * 2.0 ** -24 * dz.abs().sum(0) + edz.sum(0))
            assert (db[n:] == 7).all()


@pytest.mark.parametrize("act,act_in", [("gelu", "silu"), ("silu", "gelu_tanh"), ("gelu_tanh", "gelu")])
@pytest.mark.parametrize("T,k,n", [(3, 40, 24), (140, 33, 65)])
def test_gradients_match_differences(fpo, act, act_in, T, k, n):
    """<gradient, direction> against central differences of <dy, act(act_in(z_in) W^T + b)> in fp64,
    with a step of 1e-5: its third-order term and cancellation are below 1e-9 of the terms."""
    d = {key: t.double() for key, t in inputs("f32", T, k, n, seed=5).items()}

    def f(z_in, W, b):
        return (d["dy"] * act64(act, act64(act_in, z_in) @ W.t() + b)).sum()

    x = act64(act_in, d["z_in"])
    z = x @ d["W"].t() + d["bias"]
    dx, dW, db = (torch.empty(*s, device="cuda") for s in ((T, k), (n, k), (n,)))
    fpo.linear_vjp(d["dy"].float(), x.float(), d["W"].float(), dx, act=act_of(fpo, act), z=z.float(),
                   act_in=act_of(fpo, act_in), z_in=d["z_in"].float(), dW=dW, dbias=db)
    g = torch.Generator(device="cuda").manual_seed(T)
    h = 1e-5
    for i, grad in enumerate((dx, dW, db)):
        u = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
        args = [d["z_in"], d["W"], d["bias"]]
        lo, hi = list(args), list(args)
        lo[i], hi[i] = args[i] - h * u, args[i] + h * u
        want = (f(*hi) - f(*lo)) / (2 * h)
        # fp32 inputs (z, x: 2^-24 each), sums of up to T n k terms' roundings relative to magnitudes
        scale = (grad.double().abs() * u.abs()).sum()
        lim = ((k + n + T) * 2.0 ** -22 + 1e-8) * scale
        assert abs((grad.double() * u).sum() - want) <= lim


# rows, few tokens, single CTAs, k ranges of every tile, pair tiles with a split last wave; fp32
@pytest.mark.parametrize("dtype,T,k,n", [("bf16", 3, 264, 520), ("bf16", 20, 264, 520), ("bf16", 100, 264, 520),
                                         ("bf16", 1024, 11008, 1032), ("bf16", 384, 4096, 4096),
                                         ("bf16", 5000, 11008, 2048), ("f32", 6, 264, 520), ("f32", 70, 900, 65), ("f32", 300, 64, 132)])
def test_in_place_residual(fpo, dtype, T, k, n):
    d = inputs(dtype, T, k, n)
    y = torch.empty(T, n, dtype=DT[dtype], device="cuda")
    fpo.linear(d["x"], d["W"], y, bias=d["bias"], act=fpo.ACT_SILU, residual=d["residual"])
    r = d["residual"].clone()
    fpo.linear(d["x"], d["W"], r, bias=d["bias"], act=fpo.ACT_SILU, residual=r)
    assert torch.equal(r, y)


@pytest.mark.parametrize("dtype,T,k,n", [("bf16", 3, 4096, 1000), ("bf16", 7, 4096, 1000), ("bf16", 30, 4096, 136), ("bf16", 256, 4096, 512),
                                         ("bf16", 5000, 11008, 2048), ("f32", 70, 900, 65)])
def test_same_bits_every_time(fpo, dtype, T, k, n):
    d = inputs(dtype, T, k, n)

    def run():
        y = torch.empty(T, n, dtype=DT[dtype], device="cuda")
        dx, dW, db = torch.empty_like(d["x"]), torch.empty_like(d["W"]), torch.empty(n, device="cuda")
        fpo.linear(d["x"], d["W"], y, bias=d["bias"], act=fpo.ACT_GELU)
        fpo.linear_vjp(d["dy"], d["x"], d["W"], dx, dW=dW, dbias=db, act_in=fpo.ACT_GELU, z_in=d["z_in"])
        return y, dx, dW, db

    first = run()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))


@pytest.mark.parametrize("dtype,T", [("bf16", 9), ("bf16", 300), ("f32", 9), ("f32", 40)])
def test_nan_and_infinity_stay_in_their_rows(fpo, dtype, T):
    k, n = 136, 264
    d = inputs(dtype, T, k, n)
    y0, y = (torch.empty(T, n, dtype=DT[dtype], device="cuda") for _ in range(2))
    for act in ACTS:
        a = act_of(fpo, act)
        fpo.linear(d["x"], d["W"], y0, bias=d["bias"], act=a, residual=d["residual"])
        x, r = d["x"].clone(), d["residual"].clone()
        x[4, 5], r[7, 3], r[8, 2] = float("nan"), float("inf"), float("nan")
        fpo.linear(x, d["W"], y, bias=d["bias"], act=a, residual=r)
        assert y[4].isnan().all() and y[7, 3] == float("inf") and y[8, 2].isnan()
        y[4], y[7, 3], y[8, 2] = y0[4], y0[7, 3], y0[8, 2]
        assert torch.equal(y, y0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_activations_over_the_range_of_the_type(fpo, dtype):
    """Each activation and slope at pre-activations of every size, through a product with one."""
    mag = torch.logspace(-30, 30, 481).cuda()
    z = torch.cat([mag, -mag, torch.linspace(-20, 20, 801).cuda(), torch.zeros(1).cuda()]).to(DT[dtype])
    T = z.numel()
    x = torch.zeros(T, 8, dtype=DT[dtype], device="cuda")
    x[:, 0] = z
    W = torch.zeros(8, 8, dtype=DT[dtype], device="cuda")
    W[0, 0] = 1
    y, one = torch.empty_like(x), torch.ones_like(x)
    for act in ACTS[1:]:
        fpo.linear(x, W, y, act=act_of(fpo, act))
        want = act64(act, z.double())
        # below the smallest normal number (and near it, where a factor already was) it may be 0
        close(y[:, 0], want, HALF[dtype], 2.0 ** -17 * want.abs() + 2.0 ** -120)
        fpo.linear_vjp(one, None, W, y, act_in=act_of(fpo, act), z_in=x)
        zz = z.double().clamp(-200, 200)  # beyond, z^3 and the like would overflow in the autograd form
        close(y[:, 0], slope64(act, zz), HALF[dtype], 2.0 ** -15)


def test_no_tokens(fpo):
    for dtype in ("bf16", "f32"):
        e = lambda *s: torch.empty(*s, dtype=DT[dtype], device="cuda")  # noqa: E731
        ws = fpo.linear(e(0, 16), e(24, 16), e(0, 24))
        assert fpo.get_device_status(ws) == fpo.OK
        dW, db = torch.full((24, 16), 3.0, dtype=DT[dtype], device="cuda"), torch.full((24,), 3.0, device="cuda")
        ws = fpo.linear_vjp(e(0, 24), e(0, 16), e(24, 16), e(0, 16), dW=dW, dbias=db)
        assert fpo.get_device_status(ws) == fpo.OK
        assert (dW == 0).all() and (db == 0).all()


@pytest.mark.parametrize("T", [3, 20, 100, 260, 700])
def test_graph_replays_on_new_inputs_and_streams_do_not_mix(fpo, T):
    k, n = 1032, 520
    ins = [inputs("bf16", T, k, n, seed=s) for s in range(3)]

    class Call:
        def __init__(self):
            self.d = {key: t.clone() for key, t in ins[0].items()}
            self.y, self.dx = torch.empty_like(ins[0]["dy"]), torch.empty_like(ins[0]["x"])
            self.dW, self.db = torch.empty_like(ins[0]["W"]), torch.empty(n, device="cuda")
            self.ws = [torch.empty(max(256, s), dtype=torch.uint8, device="cuda") for s in
                       (fpo.linear_workspace(T, n, k), fpo.linear_vjp_workspace(T, n, k, act=fpo.ACT_SILU))]

        def run(self, stream=None):
            d = self.d
            fpo.linear(d["x"], d["W"], self.y, bias=d["bias"], act=fpo.ACT_GELU_TANH, workspace=self.ws[0],
                       stream=stream)
            fpo.linear_vjp(self.y, d["x"], d["W"], self.dx, act=fpo.ACT_SILU, z=d["z"], dW=self.dW,
                           dbias=self.db, workspace=self.ws[1], stream=stream)

        def out(self):
            return [t.clone() for t in (self.y, self.dx, self.dW, self.db)]

    eager = Call()
    want = []
    for d in ins:
        for key in d:
            eager.d[key].copy_(d[key])
        eager.run()
        want.append(eager.out())
    c = Call()
    c.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for d, w in zip(ins, want):
        for key in d:
            c.d[key].copy_(d[key])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(c.out(), w))
    # two calls at once, each with a workspace of its own
    calls = [Call() for _ in range(3)]
    for cc, d in zip(calls, ins):
        for key in d:
            cc.d[key].copy_(d[key])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(4):
        for cc, s in zip(calls, streams):
            cc.run(s)
    torch.cuda.synchronize()
    for cc, w in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(cc.out(), w))


@pytest.mark.parametrize("T", [20, 700])
def test_a_wait_that_runs_out_is_reported(fpo, T):
    """(No GPU fault: the wait limit is far below the time of a tile's k-blocks, 128 MB of weights in
    all, which the epilogue waits for, and every wait is bounded.)"""
    d = inputs("bf16", T, 8192, 8192)
    y, dx = torch.empty_like(d["dy"]), torch.empty_like(d["x"])

    def run():
        w1 = fpo.linear(d["x"], d["W"], y)
        w2 = fpo.linear_vjp(d["dy"], None, d["W"], dx)
        return fpo.get_device_status(w1), fpo.get_device_status(w2)

    assert run() == (fpo.OK, fpo.OK)
    y0, dx0 = y.clone(), dx.clone()
    try:
        fpo.set_wait_limit_ns(100)
        assert run() == (9, 9)  # FPO_ERR_TIMEOUT
    finally:
        fpo.set_wait_limit_ns(2_000_000_000)
    assert run() == (fpo.OK, fpo.OK)
    assert torch.equal(y, y0) and torch.equal(dx, dx0)
