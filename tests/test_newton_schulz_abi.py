"""fpo_orthogonalize_grouped and fpo_layer_muon_grouped refuse bad arguments on the host (no
GPU needed)."""
import ctypes

import pytest
import torch

OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, ARG = 0, 1, 2, 3, 4, 5, 10
P = 1 << 20   # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def fpo():
    import paper_2608_14563_gb300 as fpo
    return fpo


def ptrs(*v):
    return (ctypes.c_void_p * len(v))(*v)


def test_workspace_queries(fpo):
    q = fpo.orthogonalize_workspace
    assert q(0, 64, 64) == 0 and q(65, 64, 64) == 0 and q(1, 60, 64) == 0 and q(1, 64, 0) == 0
    assert q(1, 64, 65536 + 8) == 0 and q(1, 64, 64, 7) == 0
    # two fp16 X, one low part, fp16 A and B
    m, n = 4096, 11008
    assert 0 <= q(1, m, n) - (6 * m * n + 4 * m * m) < 8192
    assert q(1, n, m) == q(1, m, n)
    assert 0 <= q(2, m, n, fpo.F32) - 2 * (12 * m * n + 8 * m * m) < 8192
    # the update in fp32, and 16 partial norms per tile of 256 x 128
    assert 0 <= fpo.layer_muon_workspace(1, m, n) - q(1, m, n) - 4 * m * n < 8192 + m * n // 128
    assert fpo.layer_muon_workspace(1, 60, 64) == 0
    # the largest sides of the largest group fit 64 bits
    assert q(64, 65536, 65536, fpo.F32) > 64 * 20 * 65536 * 65536


def test_orthogonalize_refusals(fpo):
    need = fpo.orthogonalize_workspace(2, 64, 128)

    def call(n=2, rows=64, cols=128, dtype=1, G=ptrs(P, P), steps=5, co=None, eps=1e-7,
             O=ptrs(P, 2 * P), ws=P, size=need):
        c = None if co is None else (ctypes.c_float * len(co))(*co)
        return fpo._lib.fpo_orthogonalize_grouped(n, rows, cols, dtype, G, steps, c, eps, O, ws,
                                                  size, None)

    assert call(dtype=3) == DTYPE
    assert call(n=0) == SHAPE and call(n=65) == SHAPE
    assert call(rows=0) == SHAPE and call(cols=12) == SHAPE and call(rows=65544) == SHAPE
    assert call(steps=0) == ARG and call(steps=33) == ARG
    for eps in (0.0, -1.0, 1e-31, float("nan"), float("inf")):
        assert call(eps=eps) == ARG
    nan, inf = float("nan"), float("inf")
    assert call(steps=1, co=[nan, 0, 0]) == ARG and call(steps=1, co=[1, inf, 0]) == ARG
    assert call(steps=1, co=[0, 0, 0]) == ARG           # a bound of zero
    assert call(steps=2, co=[300, 0, 0] * 2) == ARG     # 9e4 after two steps
    assert call(steps=1, co=[7e4, -7e4, 0]) == ARG
    assert call(G=None) == NULL and call(O=None) == NULL
    assert call(G=ptrs(P, None)) == NULL and call(O=ptrs(None, P)) == NULL
    assert call(G=ptrs(P, P + 8)) == ALIGN and call(O=ptrs(P + 4, P)) == ALIGN
    assert call(ws=None) == WORKSPACE and call(size=need - 1) == WORKSPACE
    assert call(ws=P + 16) == ALIGN
    assert call(O=ptrs(P, P)) == ARG                    # one output twice


def test_muon_refusals(fpo):
    need = fpo.layer_muon_workspace(1, 64, 128)

    def call(n=1, T=16, d=64, d_ff=128, dtype=1, g=ptrs(P), A=ptrs(P), W=ptrs(P), Wo=None,
             M=ptrs(2 * P), ws=P, size=need, desc=True, **kw):
        opt = fpo.MuonDesc(*[{**dict(lr=1e-3, momentum=0.95, weight_decay=0.0, scale=1.0,
                                     eps=1e-7, nesterov=1, steps=5), **kw}[k]
                             for k in ("lr", "momentum", "weight_decay", "scale", "eps",
                                       "nesterov", "steps")], None)
        return fpo._lib.fpo_layer_muon_grouped(n, T, d, d_ff, dtype, g, A,
                                               ctypes.byref(opt) if desc else None, W, Wo, M, ws,
                                               size, None)

    assert call(desc=False) == NULL
    assert call(dtype=2) == DTYPE
    assert call(n=0) == SHAPE and call(T=-1) == SHAPE and call(T=1 << 31) == SHAPE
    assert call(d=60) == SHAPE and call(d_ff=0) == SHAPE
    for k in ("lr", "scale", "weight_decay"):
        assert call(**{k: float("nan")}) == ARG and call(**{k: float("inf")}) == ARG
    assert call(momentum=1.0) == ARG and call(momentum=-0.1) == ARG
    assert call(momentum=float("nan")) == ARG
    assert call(nesterov=2) == ARG and call(steps=0) == ARG and call(eps=0.0) == ARG
    assert call(g=None) == NULL and call(A=None) == NULL and call(W=None) == NULL
    assert call(M=None) == NULL and call(M=ptrs(None)) == NULL and call(g=ptrs(None)) == NULL
    assert call(Wo=ptrs(P + 2)) == ALIGN and call(M=ptrs(P + 4)) == ALIGN
    assert call(g=ptrs(P + 8)) == ALIGN
    assert call(size=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE
    assert call(ws=P + 128) == ALIGN
    two = fpo.layer_muon_workspace(2, 64, 128)
    assert call(n=2, g=ptrs(P, P), A=ptrs(P, P), W=ptrs(P, P), M=ptrs(2 * P, 3 * P),
                size=two) == ARG                        # one master twice
    assert call(n=2, g=ptrs(P, P), A=ptrs(P, P), W=ptrs(P, 4 * P), M=ptrs(2 * P, 2 * P),
                size=two) == ARG
    # one buffer in two arrays
    assert call(W=ptrs(2 * P)) == ARG and call(Wo=ptrs(2 * P)) == ARG and call(Wo=ptrs(P)) == ARG
    assert call(n=2, g=ptrs(P, P), A=ptrs(P, P), W=ptrs(P, 4 * P), M=ptrs(2 * P, 3 * P),
                Wo=ptrs(5 * P, P), size=two) == ARG


def test_binding_refuses_empty_and_uneven_lists(fpo):
    opt = fpo.muon_desc(lr=1e-3)
    t = torch.zeros(8, 8)
    with pytest.raises(ValueError):
        fpo.orthogonalize_grouped([], [])
    with pytest.raises(ValueError):
        fpo.orthogonalize_grouped([t], [])
    with pytest.raises(ValueError):
        fpo.layer_muon_grouped([], [], opt, [], [])
    with pytest.raises(ValueError):
        fpo.layer_muon_grouped([t, t], [t], opt, [t], [t])
    with pytest.raises(ValueError):
        fpo.layer_muon_grouped([t], [t], opt, [t], [])


def test_muon_desc_keeps_its_coefficients(fpo):
    d = fpo.muon_desc(steps=2, coeffs=[(1.5, -0.5, 0.0), (2.0, -1.5, 0.5)])
    assert [d.coeffs[i] for i in range(6)] == [1.5, -0.5, 0.0, 2.0, -1.5, 0.5]
    with pytest.raises(ValueError):
        fpo.muon_desc(steps=3, coeffs=[(1.5, -0.5, 0.0)])
