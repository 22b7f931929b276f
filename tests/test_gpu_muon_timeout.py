"""A Muon step in which a wait runs out: the status word says so, and the weights stay as they were.
(No GPU fault: the wait limit is far below the first operands' way in, and every wait is bounded.)"""
import pytest
import torch

from test_gpu_newton_schulz import DT, muon_inputs

pytestmark = pytest.mark.gpu


# the gradient's waits and the products'; T = 0 and fp32: the products' only.  (512 x 2048 bf16: one
# launch for one matrix, a launch per product for eight.)
@pytest.mark.parametrize("dtype,T,d,d_ff,n", [("bf16", 700, 512, 2048, 1), ("bf16", 700, 512, 2048, 8),
                                              ("bf16", 0, 512, 2048, 1), ("f32", 300, 257, 700, 2)])
def test_weights_are_untouched_when_a_wait_runs_out(fpo, dtype, T, d, d_ff, n):
    gs, As, W, M = muon_inputs(dtype, T, d, d_ff, n)
    opt = fpo.muon_desc(lr=1e-2, weight_decay=0.1)
    need = fpo.layer_muon_workspace(n, d, d_ff, fpo.BF16 if dtype == "bf16" else fpo.F32)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        w, m = [t.clone() for t in W], [t.clone() for t in M]
        out = [torch.full((d, d_ff), 7.0, dtype=DT[dtype], device="cuda") for _ in range(n)]
        fpo.layer_muon_grouped(gs, As, opt, w, m, W_outs=out, workspace=ws)
        return fpo.get_device_status(ws), w, m, out

    st, w0, m0, o0 = step()
    assert st == fpo.OK and all((o != 7.0).any() for o in o0)
    for _ in range(2):
        try:
            fpo.set_wait_limit_ns(100)
            st, w, m, out = step()
        finally:
            fpo.set_wait_limit_ns(2_000_000_000)
        assert st == 9  # FPO_ERR_TIMEOUT
        assert all(torch.equal(a, b) for a, b in zip(w, W))
        assert all((o == 7.0).all() for o in out)
        for a, old, new in zip(m, M, m0):
            assert ((a == old) | (a == new)).all()
    st, w, m, out = step()
    assert st == fpo.OK
    for got, want in ((w, w0), (m, m0), (out, o0)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
