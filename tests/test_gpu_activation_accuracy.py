"""The fp32 activations and slopes of the linear layer (act_math.cuh) at their own accuracy, in each
kernel that applies them.

Tolerances, u = 2^-24 (a rounding to fp32), expf 2 ulp = 4u, the MUFU reciprocal 1 ulp = 2u:
  logistic s(x) = 1 / (1 + exp(-x)): E = 4u (1 - s) + u + 2u relative, and what the argument is off by, D
  relative, times |x| (1 - s).  silu has its argument exactly; that of gelu tanh, 2 U z (1 + c z^2),
  has two rounded constants and four roundings, D = 6u.  Their values: one product more, u.
  1 - s: s off by that, and half a unit, u, of 1.  The slopes from it term by term.
  gelu: Phi(-|z|) = t Q(t) exp(-z^2 / 2) / 2.  t = 1 / d: d's fma and constant u each, the reciprocal
  2u; t Q(t) turns that into at most 2.9 times as much (|1 + t Q'/Q|, largest at z = 0).  Horner's rule
  with coefficients and steps rounded: at most 5.2u of Q.  The fit 2e-8, the exponential 4u and its
  correction u, three products 3u: added up, point by point, at most 1.34e-6, and the product with z.
  The errors average out: their mean is held to a tenth of that.
  Its slope adds z phi(z), at most 0.242, with 8u, and rounds a sum of at most 1.13."""
import math

import pytest
import torch

from test_gpu_linear import act64, act_of, slope64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -118  # near fp32's smallest normal numbers a factor may be 0
GELU = 1.34e-6
K2, C = 2 * math.sqrt(2 / math.pi), 0.044715


def grid():
    mag = torch.logspace(-12, math.log10(20.0), 20001)
    return torch.cat([torch.linspace(-20, 20, 400001), mag, -mag, torch.zeros(1)]).cuda()


def logistic_off(act, z):
    """s of the activation's argument, and what its fp32 form may be off by."""
    x = z if act == "silu" else K2 * z * (1 + C * z * z)
    s = torch.sigmoid(x)
    arg = 0 if act == "silu" else 6 * U
    return s, s * (4 * U * (1 - s) + 3 * U + x.abs() * (1 - s) * arg)


def value_limit(act, z):
    y = act64(act, z).abs()
    if act == "relu":
        return torch.zeros_like(z)
    if act == "gelu":
        return (GELU + U) * y + TINY
    s, off = logistic_off(act, z)
    return z.abs() * off * (1 + U) + U * y + TINY


def slope_limit(act, z):
    if act == "relu":
        return torch.zeros_like(z)
    val = slope64(act, z).abs()
    if act == "gelu":
        return GELU * 0.5 * torch.special.erfc(-z / math.sqrt(2)) + 0.242 * 8 * U + U * val + U
    s, off = logistic_off(act, z)
    rest = off + U                                # of 1 - s
    # silu: s (1 + z (1 - s)); gelu tanh: s + z s (1 - s) D, D = K2 (1 + 3 c z^2)
    D = torch.ones_like(z) if act == "silu" else K2 * (1 + 3 * C * z * z)
    inner = z.abs() * (1 - s) * D
    first = off * (1 + inner) + s * z.abs() * D * rest
    # a slope below fp32's numbers is 0: beyond z = -12 gelu tanh's, s(-142), is 1e-60
    return 1.01 * first + 8 * U * (s + s * inner) + U * val + TINY


def compare(got, want, lim, what):
    off = (got.double() - want).abs()
    bad = ~(off <= lim)
    assert not bad.any(), (what, (off / lim.clamp(min=1e-300))[bad].max().item(), bad.sum().item())


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("tokens", [1, 16, None], ids=["one row", "rows", "tiles"])
def test_values(fpo, act, tokens):
    z = grid()
    z = z if tokens is None else z[:: max(1, z.numel() // (200 * tokens))]
    T = z.numel()
    x = torch.zeros(T, 4, device="cuda")
    x[:, 1] = z
    W = torch.zeros(4, 4, device="cuda")
    W[2, 1] = 1
    y = torch.empty_like(x)
    for a in range(0, T, tokens or T):
        b = min(T, a + (tokens or T))
        fpo.linear(x[a:b], W, y[a:b], act=act_of(fpo, act))
    zz = z.double()
    want = act64(act, zz)
    compare(y[:, 2], want, value_limit(act, zz), act)
    if act == "gelu":  # the size of the errors, where their largest is a matter of luck
        there = want.abs() > 1e-30
        mean = ((y[:, 2].double() - want)[there] / want[there]).abs().mean().item()
        assert mean <= 0.1 * GELU, mean


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("where", ["own", "below"])
def test_slopes(fpo, act, where):
    """The layer's own activation (dZ = dY act'(Z), by the pass over dY) and the one below it (in the
    epilogue of dX)."""
    z = grid()
    T = z.numel()
    zs = torch.zeros(T, 4, device="cuda")
    zs[:, 1] = z
    W = torch.zeros(4, 4, device="cuda")
    W[1, 1] = 1
    one, dx, db = torch.ones_like(zs), torch.empty_like(zs), torch.empty(4, device="cuda")
    a = act_of(fpo, act)
    if where == "own":
        fpo.linear_vjp(one, None, W, dx, act=a, z=zs, dbias=db)
    else:
        fpo.linear_vjp(one, None, W, dx, act_in=a, z_in=zs)
    zz = z.double()
    compare(dx[:, 1], slope64(act, zz), slope_limit(act, zz), act)
