"""The workspace of a call of fpo_linear_vjp for the bias gradient alone: that of the layer, whatever
its d_in, which such a call does not read (the binding makes one up)."""
import pytest
import torch

WORKSPACE, NO_GPU = 5, (6, 7)
P = 1 << 34  # never dereferenced: validation fails first

# products of few tiles, whose parts take scratch for few columns and none for many
LAYERS = [(17, 264, 4096), (64, 4096, 4096), (300, 4096, 1024), (1000, 11008, 4096), (4096, 256, 4096),
          (8000, 4096, 11008)]


@pytest.mark.parametrize("T,n,k", LAYERS)
@pytest.mark.parametrize("act", [0, 4])
def test_the_bias_gradient_alone_takes_the_layers_workspace(T, n, k, act):
    import paper_2608_14563_gb300 as fpo
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where no call gets as far as a launch")
    z = 2 * P if act else None

    def call(d_in, size):
        return fpo._lib.fpo_linear_vjp(T, n, d_in, 1, act, P, z, None, None, 0, None, None, None, 9 * P, 10 * P,
                                       size, None)

    for d_in in (8, k):
        for layer in (8, k):
            assert call(d_in, fpo.linear_vjp_workspace(T, n, layer, 1, act)) in NO_GPU
    # the signal's copy and the ranges' sums are still asked for
    least = 256 + (T * n * 2 if act else 0)
    assert call(k, least - 1) == WORKSPACE


@pytest.mark.parametrize("T,n,k", LAYERS)
@pytest.mark.parametrize("act", [0, 4])
def test_less_than_the_outputs_need_is_refused(T, n, k, act):
    import paper_2608_14563_gb300 as fpo
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where no call gets as far as a launch")
    z = 2 * P if act else None
    need = fpo.linear_vjp_workspace(T, n, k, 1, act)

    def call(size, dx=6 * P, dw=7 * P):
        return fpo._lib.fpo_linear_vjp(T, n, k, 1, act, P, z, 3 * P, 4 * P, 0, None, dx, dw, 9 * P,
                                       10 * P, size, None)

    assert call(need) in NO_GPU and call(need - 1) == WORKSPACE
    # the larger of the two products' shares is needed with that one
    assert {call(need - 1, dx=None), call(need - 1, dw=None)} >= {WORKSPACE}


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,k", LAYERS)
def test_the_bias_gradient_alone_on_the_layers_workspace(fpo, T, n, k):
    g = torch.Generator(device="cuda").manual_seed(T + n)
    dy, z = (torch.randn(T, n, generator=g, device="cuda").bfloat16() for _ in range(2))
    for act, pre in ((fpo.ACT_NONE, None), (fpo.ACT_SILU, z)):
        size = fpo.linear_vjp_workspace(T, n, k, fpo.BF16, act)
        ws = torch.full((size + 256,), 0x5a, dtype=torch.uint8, device="cuda")
        a, b = (torch.full((n,), 7.0, device="cuda") for _ in range(2))
        fpo.linear_vjp(dy, None, None, None, act=act, z=pre, dbias=a, workspace=ws[:size])
        assert fpo.get_device_status(ws) == fpo.OK
        fpo.linear_vjp(dy, None, None, None, act=act, z=pre, dbias=b)
        assert torch.equal(a, b) and (ws[size:] == 0x5a).all()
