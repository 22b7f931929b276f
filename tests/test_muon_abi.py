"""fpo_layer_muon_grouped refuses a momentum that is also read as g or A: the gradient's kernel
writes it while it reads them (no GPU needed: the refusal comes before any use)."""
import ctypes

import pytest

WORKSPACE, ARG = 5, 10
P = 1 << 20   # never dereferenced: validation, or the workspace's size, fails first


def ptrs(*v):
    return (ctypes.c_void_p * len(v))(*v)


@pytest.fixture(scope="module")
def call():
    import paper_2608_14563_gb300 as fpo

    def call(dtype=1, T=64, g=(1, 2), A=(3, 4), W=(5, 6), Wo=(7, 8), M=(9, 10)):
        opt = fpo.muon_desc(lr=1e-3)
        arr = [None if v is None else ptrs(*[P * x for x in v]) for v in (g, A, W, Wo, M)]
        return fpo._lib.fpo_layer_muon_grouped(2, T, 64, 64, dtype, arr[0], arr[1], ctypes.byref(opt),
                                               arr[2], arr[3], arr[4], P, 256, None)
    return call


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_momentum_is_no_g_or_a(call, dtype):
    assert call(dtype) == WORKSPACE  # all arguments in order but for its size
    for M in ((1, 10), (9, 1), (2, 10), (9, 3), (4, 10)):
        assert call(dtype, M=M) == ARG


def test_what_may_be_shared(call):
    assert call(g=(1, 1), A=(3, 3)) == WORKSPACE
    assert call(g=(1, 2), A=(1, 2)) == WORKSPACE      # the Gram matrix of one input
    assert call(0, Wo=(5, 6)) == WORKSPACE            # fp32: the masters themselves
    assert call(Wo=None) == WORKSPACE
    assert call(T=0, g=(9, 5), A=(7, 6)) == WORKSPACE  # no tokens: not read
    assert call(T=0, g=None, A=None) == WORKSPACE


def test_workspace_is_what_the_header_says():
    """6 rows cols' + 4 m m' (bf16), 12 rows cols' + 8 m m' and at most 5 MB (fp32, and bf16 with a
    side of at most 64) per matrix, cols' and m' rounded up to 64; beside it 16 KB of small parts and
    their alignment."""
    import paper_2608_14563_gb300 as fpo
    for dtype in (0, 1):
        for rows, cols in ((65536, 1), (1, 65536), (33, 70), (64, 8), (767, 2049), (4096, 11008), (8, 4096),
                           (72, 136), (3000, 200), (257, 2300)):
            if dtype == 1 and (rows % 8 or cols % 8):
                continue
            m = min(rows, cols)
            split = dtype == 0 or m <= 64
            ld, ldm = -(-cols // 64) * 64, -(-m // 64) * 64
            parts = (12 if split else 6) * rows * ld + (8 if split else 4) * m * ldm
            for n in (1, 3):
                extra = fpo.orthogonalize_workspace(n, rows, cols, dtype) - n * parts
                assert 0 <= extra <= 16384 + (n * 5 * 10 ** 6 if split else 0), (dtype, rows, cols, n)
