"""Newton-Schulz orthogonalisation at the sizes of a model's layers (many waves of tiles on the
clusters), against the definition in 64 bits, and scaling by powers of two, bit for bit.  Limits as
in tests/test_gpu_newton_schulz.py."""
import pytest
import torch

from test_gpu_newton_schulz import DT, definition, limit, matrix, rel

pytestmark = pytest.mark.gpu


# (the 64-bit products of the largest are limited to two steps: 3.5e12 operations)
@pytest.mark.parametrize("dtype,rows,cols,n,steps", [("bf16", 4096, 11008, 1, 2), ("bf16", 8192, 2048, 2, 5),
                                                     ("bf16", 2600, 2600, 3, 5), ("f32", 2049, 4100, 1, 5),
                                                     ("f32", 4100, 1030, 2, 5)])
def test_layer_sizes_match_the_definition(fpo, dtype, rows, cols, n, steps):
    for kind in ("full", "rank5"):
        Gs = [matrix(rows, cols, kind, seed=l).to(DT[dtype]) for l in range(n)]
        Os = [torch.full_like(G, float("nan")) for G in Gs]
        ws = fpo.orthogonalize_grouped(Gs, Os, steps=steps)
        assert fpo.get_device_status(ws) == fpo.OK
        for G, O in zip(Gs, Os):
            assert rel(O, definition(G, steps)) < limit(dtype, kind)


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 72, 136), ("bf16", 40, 264), ("bf16", 2600, 2600),
                                             ("f32", 72, 136), ("f32", 257, 2300)])
def test_powers_of_two_change_no_bit(fpo, dtype, rows, cols):
    """Scales whose squares stay in fp32's range: sums, norm and operands scale exactly.  (Outside it the
    sums are taken in 64 bits, with one rounding less.)"""
    G = matrix(rows, cols, "full").to(DT[dtype])
    ref = torch.empty_like(G)
    fpo.orthogonalize_grouped([G], [ref], eps=1e-30)
    for e in (-40, -21, -1, 1, 40, 50):
        O = torch.empty_like(G)
        fpo.orthogonalize_grouped([G * 2.0 ** e], [O], eps=1e-30)
        assert torch.equal(O, ref), e
    want = definition(G)
    for e in (-60, 80):
        fpo.orthogonalize_grouped([G * 2.0 ** e], [ref], eps=1e-30)
        assert rel(ref, want) < limit(dtype, "full"), e
