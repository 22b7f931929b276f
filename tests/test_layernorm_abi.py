"""fpo_layernorm and fpo_layernorm_vjp refuse bad arguments on the host (no GPU needed)."""
import ctypes

import pytest

OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, ARG = 0, 1, 2, 3, 4, 5, 10
P = 1 << 20   # never dereferenced: validation fails first
MIS = P + 8


@pytest.fixture(scope="module")
def lib():
    import paper_2608_14563_gb300 as fpo
    return fpo._lib


def test_forward_refusals(lib):
    def call(T=4, d=64, dtype=1, x=P, gamma=P, beta=P, eps=1e-5, y=2 * P, mean=P, rstd=3 * P):
        return lib.fpo_layernorm(T, d, dtype, x, gamma, beta, eps, y, mean, rstd, None)

    assert call(dtype=2) == DTYPE
    assert call(T=-1) == SHAPE and call(d=0) == SHAPE and call(d=60) == SHAPE
    assert call(T=1 << 31) == SHAPE and call(d=(1 << 29) + 8) == SHAPE
    assert call(eps=-1e-5) == ARG and call(eps=float("nan")) == ARG
    assert call(x=None) == NULL and call(y=None) == NULL
    for k in ("x", "gamma", "beta", "y", "mean", "rstd"):
        assert call(**{k: MIS}) == ALIGN
    assert call(y=P) == ARG  # in place
    assert call(mean=8 * P, rstd=8 * P) == ARG


def test_backward_refusals(lib):
    need = lib.fpo_layernorm_vjp_workspace(4000, 64, 1)
    assert need > 0

    def call(T=4000, d=64, dtype=1, g=P, x=2 * P, gamma=P, eps=1e-5, min_rms=0.5, out=3 * P, dg=4 * P,
             db=5 * P, ws=P, n=need):
        return lib.fpo_layernorm_vjp(T, d, dtype, g, x, gamma, eps, min_rms, out, dg, db, ws,
                                     ctypes.c_size_t(n), None)

    assert call(dtype=-1) == DTYPE
    assert call(T=-1) == SHAPE and call(d=0) == SHAPE and call(d=12) == SHAPE
    assert call(eps=-1.0) == ARG and call(min_rms=-0.1) == ARG
    assert call(min_rms=float("nan")) == ARG
    assert call(g=None) == NULL and call(x=None) == NULL
    assert call(out=None, dg=None, db=None) == NULL
    for k in ("g", "x", "gamma", "out", "dg", "db"):
        assert call(**{k: MIS}) == ALIGN
    assert call(out=P) == ARG and call(out=2 * P) == ARG and call(db=4 * P) == ARG
    assert call(ws=None) == WORKSPACE and call(n=need - 1) == WORKSPACE
    assert call(ws=P + 16) == ALIGN


def test_workspace_query(lib):
    q = lib.fpo_layernorm_vjp_workspace
    assert q(-1, 64, 1) == 0 and q(4, 60, 1) == 0 and q(4, 64, 5) == 0 and q(4, 0, 0) == 0
    # short batches need none
    assert q(0, 4096, 1) == 0 and q(1, 4096, 1) == 0 and q(200, 256, 1) == 0 and q(1, 64, 0) == 0
    # two rows of d sums per block, at most as many blocks as rows
    assert q(128, 4096, 1) >= 128 * 2 * 4096 * 4
    assert q(16384, 4096, 1) <= 608 * 2 * 4096 * 4 + 512
    # long rows: the statistics of every row too
    assert q(1000, 20000, 0) >= 1000 * 8 + 64 * 2 * 20000 * 4
