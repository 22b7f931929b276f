"""An error that the caller's own runtime call left pending is neither cleared nor reported by the calls
and size queries of the linear layer, its backward pass and AdamW, nor by error_signal's size query."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

INVALID_DEVICE = 101  # cudaErrorInvalidDevice


def _call(fpo, name):
    """A call with every buffer in hand, and the tensors it writes."""
    g = torch.Generator(device="cuda").manual_seed(1)
    kind, *size = name.split("-")
    if kind in ("linear", "vjp"):
        dtype = torch.bfloat16 if size[0] == "bf16" else torch.float32
        T, n, k = (int(s) for s in size[1:])
        r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
        x, W, y, b = r(T, k), r(n, k), r(T, n), r(n)
        code = fpo.BF16 if size[0] == "bf16" else fpo.F32
        if kind == "linear":
            ws = torch.empty(fpo.linear_workspace(T, n, k, code), dtype=torch.uint8, device="cuda")
            return lambda: fpo.linear(x, W, y, bias=b, act=fpo.ACT_SILU, workspace=ws), [y]
        ws = torch.empty(fpo.linear_vjp_workspace(T, n, k, code, fpo.ACT_SILU), dtype=torch.uint8, device="cuda")
        dx, dW, db, z = r(T, k), r(n, k), torch.zeros(n, device="cuda"), r(T, n)
        return lambda: fpo.linear_vjp(y, x, W, dx, act=fpo.ACT_SILU, z=z, dW=dW, dbias=db, workspace=ws), [dx, dW, db]
    n = 3000
    f = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    if kind == "values":
        codes, scale = torch.arange(n, device="cuda").to(torch.uint8), torch.ones(12, device="cuda")
        out = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
        return lambda: fpo.adamw_state_values(codes, scale, out), [out]
    clip = int(size[1])
    G, W, m, v, kw = f(), f(), f(), f().square(), {}
    if size[0] == "8":
        m, v = torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
        kw = dict(scales1=[torch.zeros(12, device="cuda")], scales2=[torch.zeros(12, device="cuda")])
    ws = torch.empty(max(256, fpo.adamw_workspace([n], clip)), dtype=torch.uint8, device="cuda")
    opt = fpo.optimizer_desc(clip=clip)
    return (lambda: fpo.adamw_grouped([G], opt, [W], [m], [v], workspace=ws if clip else None, **kw)), [W, m, v]


def _leave_pending(fpo):
    """An error of the host's: no such device.  The library's own handle finds the runtime it uses."""
    assert fpo._lib.cudaGetLastError() == 0
    assert fpo._lib.cudaSetDevice(1 << 20) == INVALID_DEVICE
    assert fpo._lib.cudaPeekAtLastError() == INVALID_DEVICE


# rows, few tokens, single CTAs, pair tiles with split tiles; fp32 rows and tiles; each launch of AdamW
CALLS = ["linear-bf16-1-264-520", "linear-bf16-20-264-520", "linear-bf16-100-264-520", "linear-bf16-384-4096-4096",
         "linear-f32-6-264-520", "linear-f32-70-65-900", "vjp-bf16-20-264-520", "vjp-bf16-200-264-520",
         "vjp-f32-70-65-900", "adamw-32-0", "adamw-32-1", "adamw-32-2", "adamw-8-0", "adamw-8-1", "adamw-8-2", "values"]


@pytest.mark.parametrize("name", CALLS)
def test_a_callers_pending_error_stays(fpo, name):
    call, outs = _call(fpo, name)
    call()  # a kernel's first launch on the device sets it up
    torch.cuda.synchronize()
    again, want = _call(fpo, name)
    call2, got = _call(fpo, name)
    again()
    torch.cuda.synchronize()
    _leave_pending(fpo)
    try:
        call2()  # raises if it took the error for its own
        assert fpo._lib.cudaPeekAtLastError() == INVALID_DEVICE
    finally:
        fpo._lib.cudaGetLastError()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_size_queries_leave_it(fpo):
    es = fpo.error_signal_desc(16384, 4096, 32768)
    queries = [lambda: fpo.linear_workspace(300, 4096, 4096), lambda: fpo.linear_vjp_workspace(300, 4096, 4096),
               lambda: fpo.error_signal_workspace(es)]
    for query in queries:
        query()
        _leave_pending(fpo)
        try:
            assert query() > 0
            assert fpo._lib.cudaPeekAtLastError() == INVALID_DEVICE
        finally:
            fpo._lib.cudaGetLastError()
