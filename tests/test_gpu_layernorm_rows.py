"""Rows whose first elements say little about their mean: the statistics keep fp32's digits in every
form of the LayerNorm kernels.

A sum of squares of d terms goes through chains of at most d / 64 additions in a lane (pairs of a
vector's elements in two accumulators, 32 lanes), whose running sum is half the final one on average,
and 6 more: (d / 128 + 8) 2^-24 of the variance, half of that of 1 / sigma.  What is left of the
distance from the statistics' origin to the mean costs at most a factor of 4 of the part it enters
(only rows near their origin keep it; here every row is far off, so its second pass is around its mean):
1 / sigma within (d / 256 + 8) 2^-24, and xhat, g_out and dgamma, which have one or two such factors and
sums of their own beside it, within three times that."""
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-5


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


# T = 4096 and 300: the stream kernels (forward from 4096 on); T = 100: the register kernels
@pytest.mark.parametrize("T,d", [(4096, 5000), (4096, 8160), (300, 8192), (100, 8160)])
@pytest.mark.parametrize("start", [100.0, -1000.0])
def test_rows_with_a_shifted_start(fpo, T, d, start):
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(T, d, generator=gen, device="cuda")
    x[:, :128] += start
    g = torch.randn(T, d, generator=gen, device="cuda")
    y, out = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(T, device="cuda") for _ in range(2))
    dg = torch.empty(d, device="cuda")
    fpo.layernorm(x, None, None, y, eps=EPS, mean_out=mean, rstd_out=rstd)
    fpo.layernorm_vjp(g, x, None, out, eps=EPS, min_rms=0.0, dgamma=dg)
    X, u = x.double(), g.double()
    mu = X.mean(1, keepdim=True)
    sigma = ((X - mu) ** 2).mean(1, keepdim=True).add(EPS).sqrt()
    xh = (X - mu) / sigma
    want = (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True)) / sigma
    lim = (d / 256 + 8) * 2.0 ** -24
    assert rel(rstd, 1 / sigma[:, 0]) < lim
    assert rel(y, xh) < 3 * lim
    assert rel(out, want) < 3 * lim
    assert rel(dg, (u * xh).sum(0)) < 3 * lim


def test_constant_and_two_valued_rows(fpo):
    """A constant row gives beta and a zero signal but for sigma = sqrt(eps); a row of two values, in
    halves, has sigma = half their distance."""
    for T, d in ((4096, 5000), (300, 8192)):
        x = torch.full((T, d), 3.3, device="cuda")
        y = torch.empty_like(x)
        fpo.layernorm(x, None, None, y, eps=EPS)
        assert y.abs().max() <= 3.3 * 2.0 ** -23 / EPS ** 0.5  # mu within a rounding of 3.3
        x[:, :d // 2] = 1000.0
        x[:, d // 2:] = 1000.5
        rstd = torch.empty(T, device="cuda")
        fpo.layernorm(x, None, None, y, eps=EPS, rstd_out=rstd)
        want = 1 / (0.25 ** 2 + EPS) ** 0.5
        # the mean, 1000.25, is exact to 2^-14: a share of (2^-15)^2 / 0.0625 of the variance
        assert ((rstd.double() - want).abs() < 1e-6 * want).all()
