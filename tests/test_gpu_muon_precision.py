"""The momentum of the bf16 Muon step is a state in fp32: its gradient G = g^T A against 64 bits.

The tensor core truncates its fp32 sums: every 16-deep step of the tokens loses up to 2^-23 of the
running sum.  The sums leave the accumulator every 512 tokens, 32 steps, and are added with one
rounding each (2^-24 of the sum so far).  With R = ceil(T / 512) such additions:
products of one sign: the running sum of 32 steps is half its last value on average, 16 * 2^-23
  altogether; the sum so far is half the last on average, R / 2 * 2^-24;
products of random signs: the running sum of a run grows like the square root of its steps, 2 / 3 of
  its last value on average, 32 * 2 / 3 * 2^-23 of each run's sum.  The runs' sums are independent,
  so are their errors: the same share of the whole.  Rounding adds (sqrt(R) + 2) 2^-24."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def gradient_error(fpo, g, A):
    W, M = (torch.zeros(g.shape[1], A.shape[1], device="cuda") for _ in range(2))
    ws = fpo.layer_muon_grouped([g], [A], fpo.muon_desc(lr=1e-3), [W], [M])
    assert fpo.get_device_status(ws) == fpo.OK
    want = g.double().T @ A.double()
    return ((M.double() - want).norm() / want.norm()).item()


# one tile of 128 columns per pair, and 256
@pytest.mark.parametrize("d,d_ff", [(256, 520), (2056, 4104)])
@pytest.mark.parametrize("T", [513, 4096, 8193, 16384])
def test_gradient_keeps_fp32_digits(fpo, T, d, d_ff):
    gen = torch.Generator(device="cuda").manual_seed(T + d)
    R = -(-T // 512)
    g = torch.rand(T, d, generator=gen, device="cuda").bfloat16()
    A = torch.rand(T, d_ff, generator=gen, device="cuda").bfloat16()
    assert gradient_error(fpo, g, A) < 16 * 2.0 ** -23 + (R / 2 + 2) * 2.0 ** -24
    g = torch.randn(T, d, generator=gen, device="cuda").bfloat16()
    A = torch.randn(T, d_ff, generator=gen, device="cuda").bfloat16()
    assert gradient_error(fpo, g, A) < 64 / 3 * 2.0 ** -23 + (math.sqrt(R) + 2) * 2.0 ** -24
