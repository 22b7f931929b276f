"""AdamW over many tensors (fpo_adamw_grouped, fpo_adamw_state_values) against its definition in 64
bits, with moments in fp32 and in 8 bits.

Tolerances.  The moments are two fp32 operations each on terms of one sign or two: 2^-23 of the
magnitudes.  The step is a quotient, a square root and five products and sums: 2^-20 of its terms'
magnitudes; the weight one more rounding, 2^-24 of it.  The clip factor comes from fp32 sums of at most 4096
squares by trees of at most 24 additions and fp64 above: 2^-19.  8-bit codes equal the definition's but where
value and random fraction come within 1e-4 of a unit of the border (the fp32 moments' error, at
most 2^-22 of 16 units, is far below that): there the other one beside it is right too."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BLOCK = 256
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8)
# one element, a thread's 8, a block's 256, a chunk's 2048 or 4096, and around them
SIZES = [1, 7, 8, 9, 255, 256, 257, 511, 513, 1000, 2047, 2049, 4095, 4096, 4097, 9001, 65536, 70001]


def decode_m(code, scale):
    c = code.view(torch.uint8).long().cpu().numpy()
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 7.0), f / 8 * 2.0 ** -6)
    return np.where(c >= 128, -v, v) * spread(scale, len(c))


def decode_v(code, scale):
    c = code.long().cpu().numpy()
    e, f = c >> 3, c & 7
    return np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 16.0), f / 8 * 2.0 ** -15) * spread(scale, len(c))


def spread(scale, n):
    return np.repeat(scale.double().cpu().numpy(), BLOCK)[:n]


def noise(seed, step, tensor, n):
    """The 16 random bits of the first and of the second moment of each element."""
    M = 0xffffffff

    def mix(h):
        h ^= h >> 16
        h = h * 0x6A09E667 & M
        h ^= h >> 13
        h = h * 0xBB67AE85 & M
        return h ^ h >> 16

    key = mix(mix(mix(mix((seed + 0x9E3779B9) & M) ^ seed >> 32) ^ step & M) + tensor & M)
    i = np.arange(n, dtype=np.uint64)
    keys = np.array([mix(key ^ b) for b in range(-(-n // BLOCK))], dtype=np.uint64)
    h = (keys[(i // BLOCK).astype(int)] + i % BLOCK * np.uint64(0x9E3779B9)) & np.uint64(M)
    h ^= h >> np.uint64(15)
    h = h * np.uint64(0x6A09E667) & np.uint64(M)
    h ^= h >> np.uint64(16)
    return (h >> np.uint64(16)).astype(np.int64), (h & np.uint64(0xffff)).astype(np.int64)


class Tensors:
    def __init__(self, sizes, bits, seed=0, g16=None, out=None, decay=None):
        g = torch.Generator(device="cuda").manual_seed(seed + len(sizes))
        rn = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
        self.n, self.bits = sizes, bits
        self.G = [(1e-3 * torch.exp(rn(1)) * rn(n)).to(torch.bfloat16 if (k if g16 is None else g16) % 2
                                                       else torch.float32) for k, n in enumerate(sizes)]
        self.W = [0.5 * rn(n) for n in sizes]
        self.out = [None if k % 3 == 2 else torch.full((n,), 7.0, device="cuda").to(
            torch.bfloat16 if k % 3 == 0 else torch.float32) for k, n in enumerate(sizes)]
        self.decay = [0.1 * (k % 4) for k in range(len(sizes))]
        if bits == 32:
            self.m = [1e-3 * rn(n) for n in sizes]
            self.v = [(1e-3 * rn(n)) ** 2 for n in sizes]
            self.ms = self.vs = None
        else:
            self.m = [torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for n in sizes]
            self.v = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes]
            self.ms = [torch.zeros(-(-n // BLOCK), device="cuda") for n in sizes]
            self.vs = [torch.zeros(-(-n // BLOCK), device="cuda") for n in sizes]

    def step(self, fpo, t, clip=0, seed=3, stream=None, workspace=None):
        opt = fpo.optimizer_desc(fpo.OPT_ADAMW, step=t, clip=clip, clip_frac=0.004, **HYPER)
        return fpo.adamw_grouped(self.G, opt, self.W, self.m, self.v, scales1=self.ms, scales2=self.vs,
                                 W_outs=self.out, weight_decays=self.decay, seed=seed, stream=stream,
                                 workspace=workspace)

    def moments(self, k):
        if self.bits == 32:
            return [x[k].double().cpu().numpy() for x in (self.m, self.v)]
        return [decode_m(self.m[k], self.ms[k]), decode_v(self.v[k], self.vs[k])]

    def before(self):
        return [(self.G[k].double().cpu().numpy(), self.W[k].double().cpu().numpy(), *self.moments(k))
                for k in range(len(self.n))]


def definition(g, w, m, v, wd, t, clip):
    """New m, v, step, its terms' magnitudes, W and the clip factor."""
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    lr, eps, frac = (np.float32(x).astype(float) for x in (HYPER["lr"], HYPER["eps"], 0.004))
    lim, s = frac * np.linalg.norm(w), 1.0
    if clip == 2 and np.linalg.norm(g) > lim:
        g = g * (lim / np.linalg.norm(g))
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    a = m / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    d = -lr * (a + wd * w)
    if clip == 1 and np.linalg.norm(d) > lim:
        s = lim / np.linalg.norm(d)
    return m, v, s * d, lr * s * (np.abs(a) + wd * np.abs(w)), w + s * d


def check(x, before, t, clip, seed=3):
    for k, (g, w, m, v) in enumerate(before):
        wd = float(np.float32(x.decay[k]))
        m1, v1, d, terms, w1 = definition(g, w, m, v, wd, t, clip)
        # m may cancel against the new gradient: its error as a part of the step
        me = 2.0 ** -22 * (np.abs(m) + np.abs(g))
        rel = 2.0 ** -19 + (2.0 ** -18 if clip else 0)
        lim = rel * terms + HYPER["lr"] * me / (np.sqrt(np.maximum(v1, 1e-60))) * 30 + 2.0 ** -23 * np.abs(w1)
        got = x.W[k].double().cpu().numpy()
        assert (np.abs(got - w1) <= lim).all(), (k, np.max(np.abs(got - w1) / lim))
        if x.out[k] is not None:
            assert torch.equal(x.out[k].float(), x.W[k].to(x.out[k].dtype).float())
        if x.bits == 32:
            gm, gv = x.moments(k)
            c = 2.0 ** -18 if clip == 2 else 2.0 ** -22
            assert (np.abs(gm - m1) <= c * (np.abs(m) + np.abs(g)) + 1e-44).all()
            assert (np.abs(gv - v1) <= 2 * c * (v + g * g) + 1e-44).all()
        else:
            um, uv = noise(seed, t, k, len(g))
            check_codes(m1, um, x.m[k].view(torch.uint8), x.ms[k], 7, 7, True, me)
            check_codes(v1, uv, x.v[k], x.vs[k], 16, 14, False, 2.0 ** -20 * v1 + 2.0 ** -149)


def check_codes(val, u, code, scale, bias, top, signed, err):
    code = code.cpu().numpy().astype(np.int64)
    n = len(val)
    pad = -(-n // BLOCK) * BLOCK - n
    amax = np.pad(np.abs(val), (0, pad)).reshape(-1, BLOCK).max(1)
    want = 2.0 ** (np.floor(np.log2(np.maximum(amax, 2.0 ** -100))) - top)
    got = scale.double().cpu().numpy()
    border = np.abs(np.log2(np.maximum(amax, 1e-300)) % 1 - 0.5) > 0.4999  # the maximum next to a power of two
    assert ((got == want) | (border & ((got == 2 * want) | (got == want / 2)))).all()
    mag = code & 127 if signed else code
    s = np.repeat(got, BLOCK)[:n]
    y = np.abs(val) / s
    e = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), 1 - bias)
    unit = 2.0 ** (e - 3)
    place = y / unit + u / 65536
    k = np.floor(place)
    near = np.abs(place - np.round(place)) <= 1e-4 + np.abs(err) / s / unit
    low = (k + 8 * (e + bias - 1)).astype(np.int64)
    other = np.where(place - k > 0.5, low + 1, low - 1)
    ok = (mag == low) | (near & (mag == other))
    if not signed:
        # the moment is an fp32 number: (1 - beta2) g^2 under its smallest, 2^-149, is 0 or that one
        # (g = 1e-30: 1e-62), and is kept as what it then is
        ok = (mag == np.where(val > 0, np.maximum(low, 1), low)) | (near & (mag == np.maximum(other, 1)))
        ok |= (val < 2.0 ** -149) & (mag == 0)
    assert ok.all(), np.flatnonzero(~ok)[:5]
    if signed:
        assert (((code >= 128) == (val < 0)) | (np.abs(val) <= err)).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("clip", [0, 1, 2])
@pytest.mark.parametrize("sizes", [[1], [2049], SIZES, [300] * 12, [5] * 13, [257] * 131, [200000, 3, 40000]],
                         ids=["one", "odd", "sizes", "few", "many", "launches", "uneven"])
def test_steps_match_the_definition(fpo, bits, clip, sizes):
    x = Tensors(sizes, bits)
    for t in (1, 2, 3):
        before = x.before()
        x.step(fpo, t, clip)
        check(x, before, t, clip)


@pytest.mark.parametrize("n", [4096 * 7, 70001])
def test_moments_are_rounded_as_written(fpo, n):
    """Each product and sum of the new moments by itself, as any fp32 arithmetic has it."""
    for g16 in (0, 1):
        x = Tensors([n], 32, g16=g16)
        g, m, v = x.G[0].float(), x.m[0].clone(), x.v[0].clone()
        x.step(fpo, 3)
        b1, b2 = HYPER["beta1"], HYPER["beta2"]
        assert torch.equal(x.m[0], b1 * m + (1 - b1) * g) and torch.equal(x.v[0], b2 * v + (1 - b2) * g * g)


def test_empty_tensors_are_skipped(fpo):
    for bits in (32, 8):
        for clip in (0, 1):
            x = Tensors([0, 300, 0, 0, 5, 0], bits)
            before = x.before()
            x.step(fpo, 1, clip)
            for k in (1, 4):
                one = Tensors([0, 300, 0, 0, 5, 0], bits)
                assert torch.equal(one.G[k], x.G[k])
            full = [b if len(b[0]) else None for b in before]
            keep = [k for k, b in enumerate(full) if b is not None]
            for k in keep:
                g, w, m, v = before[k]
                w1 = definition(g, w, m, v, float(np.float32(x.decay[k])), 1, clip)[4]
                assert np.abs(x.W[k].double().cpu().numpy() - w1).max() <= 1e-6


@pytest.mark.parametrize("clip", [0, 1, 2])
def test_both_kinds_of_moments_in_one_call(fpo, clip):
    """The same bits as each kind has in a call of its own where its tensors keep their places."""
    sizes = [300, 5000, 1, 257, 4096, 70]
    small, large = Tensors(sizes, 8, g16=0), Tensors(sizes, 32, g16=0)
    mixed = Tensors(sizes, 32, g16=0)
    kinds = [8, 32, 8, 32, 32, 8]
    other = Tensors(sizes, 8, g16=0)
    for k, bits in enumerate(kinds):
        if bits == 8:
            mixed.m[k], mixed.v[k] = other.m[k], other.v[k]
    mixed.ms = [other.ms[k] if b == 8 else None for k, b in enumerate(kinds)]
    mixed.vs = [other.vs[k] if b == 8 else None for k, b in enumerate(kinds)]
    for x in (small, large, mixed):
        x.G, x.W = [g.clone() for g in large.G], [w.clone() for w in large.W]
    for t in (1, 2):
        for x in (small, large, mixed):
            x.step(fpo, t, clip)
    for k, bits in enumerate(kinds):
        want = small if bits == 8 else large
        for a, b in ((mixed.W, want.W), (mixed.m, want.m), (mixed.v, want.v)):
            assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), k


def test_the_step_is_that_of_the_layer_optimizer(fpo):
    """That of fpo_layer_optimize_grouped on the gradient it forms (fp32, no clip), but for roundings
    and its rates in float: 1 - 0.999f is 1.3e-5 off, 1 - 0.9f 2.4e-7, both relative."""
    T, d, f = 40, 24, 36
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    gs, A, W, m, v = rn(T, d), rn(T, f), rn(d, f), 0.1 * rn(d, f), rn(d, f) ** 2
    G = torch.empty(d, f, device="cuda")
    fpo.layer_update(gs, A, 0.0, G_out=G)
    opt = fpo.optimizer_desc(fpo.OPT_ADAMW, clip=fpo.CLIP_NONE, step=7, lr=1e-2)
    a, b = [W.clone(), m.clone(), v.clone()], [W.clone(), m.clone(), v.clone()]
    fpo.layer_optimize_grouped([gs], [A], opt, [a[0]], states1=[a[1]], states2=[a[2]])
    fpo.adamw_grouped([G], opt, [b[0]], [b[1]], [b[2]])
    rel = [((p - q).abs() / s).max().item() for p, q, s in zip(a, b, (W.abs() + 0.1, m.abs() + G.abs(), v + G * G))]
    assert rel[0] <= 1e-2 * 1e-5 * 10 and rel[1] <= 1e-6 and rel[2] <= 2e-5, rel


def test_elements_behind_a_tensor_stay(fpo):
    n, spare = 301, 40
    for clip in (0, 1):
        W = torch.full((n + spare,), 0.5, device="cuda")
        out = torch.full((n + spare,), 7.0, device="cuda", dtype=torch.bfloat16)
        m = torch.full((n + spare,), 0x55, device="cuda", dtype=torch.uint8)
        v = m.clone()
        ms, vs = (torch.full((4,), 2.0 ** -20, device="cuda") for _ in range(2))
        opt = fpo.optimizer_desc(clip=clip, step=1)
        fpo.adamw_grouped([torch.ones(n, device="cuda")], opt, [W[:n]], [m[:n].view(torch.float8_e4m3fn)],
                          [v[:n]], scales1=[ms[:2]], scales2=[vs[:2]], W_outs=[out[:n]])
        assert (W[n:] == 0.5).all() and (out[n:] == 7).all() and (m[n:] == 0x55).all() and (v[n:] == 0x55).all()
        assert (ms[2:] == 2.0 ** -20).all() and (vs[2:] == 2.0 ** -20).all()
        assert (W[:n] != 0.5).all() and (out[:n] != 7).all()


def test_same_bits_every_time_and_other_seeds_round_otherwise(fpo):
    def run(seed, t=2):
        x = Tensors([5000, 700], 8)
        x.step(fpo, 1, 1, seed=seed)
        x.step(fpo, t, 1, seed=seed)
        return x.W + [c.view(torch.uint8) for c in x.m] + x.v + x.ms + x.vs

    a = run(5)
    assert all(torch.equal(p, q) for p, q in zip(a, run(5)))
    for other in (run(6), run(5 + (1 << 40)), run(5, t=3)):
        assert (a[2] != other[2]).float().mean() > 0.1 and (a[4] != other[4]).float().mean() > 0.1


def test_rounding_keeps_the_expected_value(fpo):
    """Elements of one value, rounded with each one's own bits: the mean is the value, to five
    standard deviations of a mean of n (a deviation is at most half a unit, a unit 1/8 of the value)."""
    n = 1 << 20
    for value in (1e-4, 1.37e-3, 0.9):
        x = Tensors([n], 8)
        x.G[0] = torch.full((n,), value, device="cuda")
        x.step(fpo, 1)
        m, v = x.moments(0)
        lim = 5 * 0.5 / 8 / math.sqrt(n) + 2.0 ** -16
        b1, b2 = HYPER["beta1"], HYPER["beta2"]
        g = float(np.float32(value))
        assert abs(m.mean() / ((1 - b1) * g) - 1) <= lim and abs(v.mean() / ((1 - b2) * g * g) - 1) <= lim
        assert len(np.unique(m)) == 2 and len(np.unique(v)) == 2


def test_second_moments_fall_without_gradients(fpo):
    """By beta2 a step in the mean, though a code's unit is ten times that: after 60 steps without a
    gradient 0.99^60 is left, to five deviations (each step adds at most a unit's worth of variance
    p (1 - p) u^2 <= 0.01 / (1/16) (1/8)^2)."""
    n = 1 << 16
    x = Tensors([n], 8)
    x.step(fpo, 1)
    v0 = x.moments(0)[1]
    x.G[0] = torch.zeros(n, device="cuda")
    for t in range(2, 62):
        x.step(fpo, t)
    big = v0 > v0.max() / 16  # far from the format's lowest code
    left = x.moments(0)[1][big].sum() / v0[big].sum()
    sd = math.sqrt(60 * 0.16 / 64 / big.sum() * (v0[big] ** 2).mean()) / v0[big].mean()
    assert abs(left / 0.99 ** 60 - 1) <= 5 * sd + 1e-3


def test_second_moments_of_nonzero_gradients_are_never_zero(fpo):
    n = 4096
    x = Tensors([n], 8)
    g = torch.full((n,), 1e-6, device="cuda")
    g[::BLOCK] = 1e3      # the block's scale is far above the others
    g[5::BLOCK] = 0.0
    x.G[0] = g
    x.step(fpo, 1)
    v = x.v[0].cpu().numpy()
    assert (v[5::BLOCK] == 0).all() and (np.delete(v.reshape(-1, BLOCK), 5, 1) > 0).all()
    w = x.W[0].clone()
    x.G[0] = torch.zeros(n, device="cuda")
    x.step(fpo, 2)
    # what is kept of the tiny gradients cannot move a weight by more than a few rates: the kept m is
    # at most 2^-9 scales' unit above the truth, sqrt(v) at least its lowest code's
    assert (x.W[0] - w).abs().max() <= 30 * HYPER["lr"]


@pytest.mark.parametrize("bits", [32, 8])
def test_nan_and_infinity(fpo, bits):
    n = 1024
    for bad in (float("nan"), float("inf"), -float("inf")):
        x, ref = Tensors([n], bits, g16=0), Tensors([n], bits, g16=0)
        x.G[0][300] = bad
        x.step(fpo, 1)
        ref.step(fpo, 1)
        ok = torch.ones(n, dtype=torch.bool, device="cuda")
        ok[300] = False
        assert torch.equal(x.W[0][ok], ref.W[0][ok])
        m, v = x.moments(0)
        rm, rv = ref.moments(0)
        keep = np.ones(n, bool)
        keep[256:512] = bits == 32
        keep[300] = False
        assert np.array_equal(m[keep], rm[keep]) and np.array_equal(v[keep], rv[keep])
        assert not np.isfinite(v[300]) and not np.isfinite(m[300])
        if bits == 8:
            assert np.isnan(m[256:512]).all() and np.isnan(v[256:512]).all()


def test_an_infinite_gradient_under_the_clip(fpo):
    """On the gradient the norm is infinite and the factor 0: the other elements see no gradient.  On
    the step the norm is NaN (infinity by infinity) and the factor 1."""
    for clip in (1, 2):
        x = Tensors([1024], 32, g16=0)
        x.G[0][300] = float("inf")
        g, w, m, v = x.before()[0]
        x.step(fpo, 1, clip)
        if clip == 2:
            g = 0 * np.where(np.isfinite(g), g, 0)
        g = np.where(np.isfinite(g), g, 0)
        m1, v1, _, _, w1 = definition(g, w, m, v, 0.0, 1, 0)
        ok = np.arange(1024) != 300
        gm, gv = x.moments(0)
        # (m is a difference where the signs differ: 2^-22 of both terms, as in check())
        assert (np.abs(gm - m1) <= 2.0 ** -22 * (np.abs(m) + np.abs(g)))[ok].all()
        assert np.allclose(gv[ok], v1[ok], rtol=1e-6, atol=0)
        assert np.allclose(x.W[0].double().cpu().numpy()[ok], w1[ok], rtol=0, atol=1e-6)
        assert not np.isfinite(gm[300])


def test_zero_blocks_and_extreme_sizes(fpo):
    """Moments over the range of fp32: scales stay in range, values within a unit."""
    n = 2560
    x = Tensors([n], 8)
    x.G[0] = torch.zeros(n, device="cuda")
    for k, mag in enumerate((0.0, 1e-30, 1e-18, 1e-10, 1e-3, 1.0, 1e6, 1e15, 3e18, 1e-38)):
        x.G[0][256 * k:256 * (k + 1)] = mag * torch.linspace(0.5, 1, 256, device="cuda")
    before = x.before()
    x.step(fpo, 1)
    check(x, before, 1, 0)
    m, _ = x.moments(0)
    assert (m[:256] == 0).all()


def test_state_values(fpo):
    for dtype in (torch.float32, torch.bfloat16):
        for n in (1, 8, 255, 256, 1027, 5000):
            codes = (torch.arange(n, device="cuda") * 37 % 256).to(torch.uint8)
            scale = 2.0 ** torch.arange(-20, -20 + -(-n // BLOCK), device="cuda").float()
            out = torch.full((n + 9,), 7.0, device="cuda", dtype=dtype)
            fpo.adamw_state_values(codes, scale, out[:n])
            assert np.array_equal(out[:n].double().cpu().numpy(), decode_v(codes, scale))
            assert (out[n:] == 7).all()
            m = torch.where((codes & 127) == 127, codes - 1, codes).view(torch.float8_e4m3fn)  # (no NaN codes)
            fpo.adamw_state_values(m, scale, out[:n])
            want = decode_m(m, scale)
            assert np.array_equal(out[:n].double().cpu().numpy(), want)
            assert np.array_equal(m.float().double().cpu().numpy() * spread(scale, n), want)
            assert (out[n:] == 7).all()


def test_graphs_and_streams(fpo):
    for bits in (32, 8):
        for clip in (0, 1):
            want, got = Tensors(SIZES, bits), Tensors(SIZES, bits)
            ws = torch.empty(max(256, fpo.adamw_workspace(SIZES, clip)), dtype=torch.uint8, device="cuda")
            want.step(fpo, 4, clip)
            want.step(fpo, 4, clip)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            got.step(fpo, 4, clip, stream=s)
            torch.cuda.current_stream().wait_stream(s)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got.step(fpo, 4, clip, workspace=ws)
            graph.replay()
            for a, b in zip(want.W + want.m + want.v, got.W + got.m + got.v):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_offsets_beyond_32_bits(fpo):
    """A tensor of more than 2^31 elements: its last elements as a small tensor's with the same bits."""
    n, tail = (1 << 31) + 4096 + 5, 4096 + 5
    G = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    G[-tail:] = 1e-3 * torch.randn(tail, device="cuda")
    W = torch.zeros(n, device="cuda")
    W[-tail:] = torch.randn(tail, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = (torch.zeros(-(-n // BLOCK), device="cuda") for _ in range(2))
    w0 = W[-tail:].clone()
    opt = fpo.optimizer_desc(clip=fpo.CLIP_NONE, step=1, **HYPER)
    fpo.adamw_grouped([G], opt, [W], [m.view(torch.float8_e4m3fn)], [v], scales1=[ms], scales2=[vs])
    w, g = w0.double().cpu().numpy(), G[-tail:].double().cpu().numpy()
    _, _, d, _, w1 = definition(g, w, 0 * g, 0 * g, 0.01, 1, 0)
    assert np.abs(W[-tail:].double().cpu().numpy() - w1).max() <= 1e-6 * np.abs(w1).max()
    assert (W[:1000] == 0).all() and (v[:-tail] == 0).all()
    first = n - tail
    assert first % BLOCK == 0
    val = decode_m(m[first:], ms[first // BLOCK:])
    assert np.abs(val - 0.1 * g).max() <= 0.1 * np.abs(g).max() / 8
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    fpo.adamw_state_values(m.view(torch.float8_e4m3fn), ms, out)
    assert np.array_equal(out[first:].double().cpu().numpy(), val) and (out[:first] == 0).all()
