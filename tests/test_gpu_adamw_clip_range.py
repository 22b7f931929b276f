"""The relative clip of fpo_adamw_grouped where the squares of weights, gradients or steps leave fp32's
range, against its definition in 64 bits (the clip factor 1 or 0 that inf / inf, 0 / 0 and x / inf would
give is wrong by many orders).

Tolerances.  A norm's sum of squares: 16 products and additions of a thread, 5 of its warp, 8 of the
block's, 2^-24 each, and the word that holds it, 2^-21: 2.4 x 2^-20, of the norm half of that.  The
factor is a quotient of two norms: 2.4 x 2^-20 and its own rounding, 2^-24.  m takes three more
roundings: 2^-18 in all; v the factor twice: 2^-17.  A step is a quotient with two MUFU operations, 2^-21, of
moments with those errors, which it takes the quotient of: 2^-17 of its terms; the weight one more
rounding, 2^-24 of it."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import BLOCK

pytestmark = pytest.mark.gpu

BETA1, BETA2, EPS, FRAC = 0.9, 0.99, 1e-8, 0.004


def definition(g, w, wd, lr, clip):
    """A first step from zero moments: the factor, m, v, W and the magnitudes of the step's terms."""
    lim, s = float(np.float32(FRAC)) * np.linalg.norm(w), 1.0
    gs = g
    if clip == 2 and np.linalg.norm(g) > lim:
        gs = g * (lim / np.linalg.norm(g))
    m, v = (1 - BETA1) * gs, (1 - BETA2) * gs * gs
    a = gs / (np.abs(gs) + float(np.float32(EPS)))
    d = -lr * (a + wd * w)
    if clip == 1 and np.linalg.norm(d) > lim:
        s = lim / np.linalg.norm(d)
    return m, v, w + s * d, lr * s * (np.abs(a) + wd * np.abs(w))


def tensors(n, w_mag, g_mag):
    """Magnitudes are a number, or (a number, one for the elements of every third warp of 32 x 8)."""
    g = torch.Generator(device="cuda").manual_seed(n)

    def make(mag):
        x = torch.randn(n, generator=g, device="cuda")
        if not isinstance(mag, tuple):
            return mag * x
        third = torch.arange(n, device="cuda") // BLOCK % 3 == 1
        return torch.where(third, mag[1] * x, mag[0] * x)

    return make(w_mag), make(g_mag)


def step(fpo, W, G, bits, clip, lr, wd):
    W, n = W.clone(), W.numel()
    kw = {}
    if bits == 32:
        m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    else:
        m = torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda")
        v = torch.zeros(n, dtype=torch.uint8, device="cuda")
        kw = dict(scales1=[torch.zeros(-(-n // BLOCK), device="cuda")],
                  scales2=[torch.zeros(-(-n // BLOCK), device="cuda")])
    opt = fpo.optimizer_desc(fpo.OPT_ADAMW, lr=lr, beta1=BETA1, beta2=BETA2, eps=EPS, clip=clip, clip_frac=FRAC)
    fpo.adamw_grouped([G], opt, [W], [m], [v], weight_decays=[wd], **kw)
    return W, m, v


# gradients that would be dropped; that would not be clipped; weights whose own squares overflow or vanish;
# chunks and warps of each kind beside one another; what is in range as it was
@pytest.mark.parametrize("n", [1, 300, 2049, 70001])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w_mag,g_mag", [(0.5, 1e20), (0.5, 1e30), (1e20, 1e21), (1e-24, 1e-25), (1e-30, 1e-31),
                                         (0.5, (1e20, 1e-25)), ((0.5, 1e-22), (1e-3, 1e-20)), ((1e13, 1e-3), 1e12),
                                         ((1e-30, 1e-18), 1e-17), (0.5, 1.0)])
def test_clip_on_the_gradient(fpo, n, bits, w_mag, g_mag):
    lr, wd = 1e-3 * max(w_mag if isinstance(w_mag, tuple) else (w_mag,)), 0.0
    W, G = tensors(n, w_mag, g_mag)
    w1, m1, v1 = step(fpo, W, G, bits, 2, lr, wd)
    w, g = W.double().cpu().numpy(), G.double().cpu().numpy()
    m, v, want, terms = definition(g, w, wd, float(np.float32(lr)), 2)
    if bits == 32:
        tiny = 2.0 ** -148  # fp32's smallest numbers: a product and a sum
        assert (np.abs(m1.double().cpu().numpy() - m) <= 2.0 ** -18 * np.abs(m) + tiny).all()
        assert (np.abs(v1.double().cpu().numpy() - v) <= 2.0 ** -17 * v + tiny).all()
    # (v below 2^-126 counts as 0 in the square root: sqrt(v / (1 - beta2)) is then below 2^-59, beside eps)
    err = np.abs(w1.double().cpu().numpy() - want)
    lim = (2.0 ** -17 + 2.0 ** -59 / EPS) * terms + 2.0 ** -24 * np.abs(want) + 2.0 ** -148
    assert (err <= lim).all(), np.max(err / lim)


@pytest.mark.parametrize("n", [1, 300, 2049, 70001])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w_mag,lr,wd", [(1e20, 10.0, 0.1), (1e25, 1.0, 1.0), ((1e20, 1e-3), 10.0, 0.1),
                                         (1e-24, 1e-25, 0.0), ((1e-24, 1e-20), 1e-22, 0.0), (0.5, 0.1, 0.1)])
def test_clip_on_the_step(fpo, n, bits, w_mag, lr, wd):
    W, G = tensors(n, w_mag, 1e-3)
    w1, m1, v1 = step(fpo, W, G, bits, 1, lr, wd)
    w, g = W.double().cpu().numpy(), G.double().cpu().numpy()
    _, _, want, terms = definition(g, w, float(np.float32(wd)), float(np.float32(lr)), 1)
    err = np.abs(w1.double().cpu().numpy() - want)
    lim = 2.0 ** -17 * terms + 2.0 ** -23 * np.abs(want) + 2.0 ** -148
    assert (err <= lim).all(), np.max(err / lim)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("clip,g_mag,lr", [(1, 1e-3, 1e-25), (1, 1e-3, 1e-3), (2, 1e-25, 1e-3), (2, 1e-38, 1e-3),
                                           (2, 1.0, 1e-3), (2, 1e30, 1e-3)])
def test_a_tensor_of_zeros_does_not_move(fpo, bits, clip, g_mag, lr):
    for n in (1, 300, 5000):
        W, G = tensors(n, 0.0, g_mag)
        w1, m1, v1 = step(fpo, W, G, bits, clip, lr, 0.0)
        assert (w1 == 0).all()
        if clip == 2:
            assert (m1.float() == 0).all() and (v1.float() == 0).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("clip", [1, 2])
def test_a_nan_among_them_leaves_the_others_unclipped(fpo, bits, clip):
    """The norm is NaN, and the factor 1."""
    W, G = tensors(5000, 0.5, (1e-3, 1e-25))
    G[700] = float("nan")
    clipped, free = step(fpo, W, G, bits, clip, 1e-3, 0.0), step(fpo, W, G, bits, 0, 1e-3, 0.0)
    for a, b in zip(clipped, free):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert clipped[0].isnan().sum() == 1
