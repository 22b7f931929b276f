"""LayerNorm's kernels for large batches when their waits run out (no GPU fault: every wait is
bounded, here by a nanosecond).  Some of the backward pass's waits, for rows that are still on their
way or whose statistics another warp forms, surely outlast that; the forward pass's may."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,T,d", [(torch.bfloat16, 16384, 8192), (torch.float32, 4100, 5000)])
def test_what_was_not_reached_is_nan(fpo, dtype, T, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, g = (torch.randn(T, d, generator=gen, device="cuda").to(dtype) for _ in range(2))

    def call():
        y, out = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        dg, db = (torch.full((d,), 7.0, device="cuda") for _ in range(2))
        fpo.layernorm(x, None, None, y)
        fpo.layernorm_vjp(g, x, None, out, dgamma=dg, dbeta=db)
        torch.cuda.synchronize()
        return y, out, dg, db

    want = call()
    assert not any(t.isnan().any() or (t == 7.0).all() for t in want)
    try:
        fpo.set_wait_limit_ns(1)
        short = call()
    finally:
        fpo.set_wait_limit_ns(2_000_000_000)
    y, out, dg, db = short
    assert out.isnan().any() and dg.isnan().any() and db.isnan().any()
    for a, b in zip(want, short):  # right, or NaN: nothing is left as it was
        assert (b.isnan() | (a == b)).all()
    # a block gives up for good: the columns of its later rows are NaN too, in the weight sums as well
    assert (dg.isnan() == db.isnan()).all()
    lost = out.isnan().any(0)
    assert (dg.isnan() == lost).all()
    assert all(torch.equal(a, b) for a, b in zip(want, call()))
