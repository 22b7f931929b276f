"""The bounds of the singular values that the Newton-Schulz products' operands are scaled by, against
dense scans of the polynomials (no GPU needed), and steps whose polynomials have a tiny leading
coefficient.

A bound that misses an interior maximum lets the scaled matrices leave fp16's range, or refuses
coefficients whose polynomial ends near zero."""
import ctypes
import random

import numpy as np
import pytest
import torch

ARG, WORKSPACE = 10, 5


@pytest.fixture(scope="module")
def lib():
    import paper_2608_14563_gb300 as fpo
    fn = fpo._lib.fpo_testing_ns_bounds
    fn.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_double)]
    fn.restype = None
    return fpo


def bounds(lib, *triples):
    flat = [v for t in triples for v in t]
    co, out = (ctypes.c_float * len(flat))(*flat), (ctypes.c_double * len(triples))()
    lib._lib.fpo_testing_ns_bounds(len(triples), co, out)
    return list(out)


def check(got, a, b, c, u):
    """The maximum of a grid is at most the bound, and below it by no more than the curvature over a
    grid step allows (and the rounding of the sums)."""
    a, b, c = (float(np.float32(v)) for v in (a, b, c))
    n = 20001
    s = np.linspace(0.0, u, n)
    scan = np.abs(s * (a + s * s * (b + s * s * c))).max()
    terms = abs(a) * u + abs(b) * u ** 3 + abs(c) * u ** 5
    step = u / (n - 1)
    slack = (6 * abs(b) * u + 20 * abs(c) * u ** 3) * step ** 2 / 8 + 1e-14 * terms
    assert scan - 1e-14 * terms <= got <= scan + slack, (a, b, c, u, got, scan)


TINY = [0.0] + [s * 10.0 ** -e for e in (0, 2, 4, 6, 8, 12, 16, 20, 30, 40) for s in (1.0, -1.0)]


@pytest.mark.parametrize("c", TINY)
def test_bound_of_cubics_and_near_cubics(lib, c):
    for a, b in ((1.0009765625, -1.0), (2.6, -2.574), (1.5, -0.5), (1.0, -1.0), (-1.0, 1.5),
                 (3.4445, -4.775), (1e-20, -1.0), (0.0, 1.0), (1.0, 1e-20), (1.0, 0.0)):
        check(bounds(lib, (a, b, c))[0], a, b, c, 1.0)


def test_bound_of_any_polynomials(lib):
    rng = random.Random(4)

    def coef():
        return rng.choice([-1, 1]) * 10.0 ** rng.uniform(-10, 3) if rng.random() < 0.9 else 0.0

    for _ in range(3000):
        first, second = [coef() for _ in range(3)], [coef() for _ in range(3)]
        b = bounds(lib, first, second)
        check(b[0], *first, 1.0)
        if 1e-30 < b[0] < 1e30:
            check(b[1], *second, b[0])


@pytest.mark.parametrize("co", [(1.0, -1.0, 1e-20), (1.0, -1.0, 0.0), (2.6, -2.6, 1e-30)])
def test_polynomials_that_end_at_zero_are_taken(lib, co):
    P = 1 << 20  # never dereferenced: the workspace is too small
    ptr = (ctypes.c_void_p * 1)(P)
    rc = lib._lib.fpo_orthogonalize_grouped(1, 64, 128, 1, ptr, 1, (ctypes.c_float * 3)(*co), 1e-7,
                                            ptr, P, 256, None)
    assert rc == WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("first", [(1.0009765625, -1.0, 1e-20), (2.6, -2.574, 1e-20)])
def test_steps_with_a_tiny_leading_coefficient(fpo, dtype, first):
    """Three equal singular values, 1 / sqrt 3 of the norm each: where s - s^3 is largest.  The
    limits are those of tests/test_gpu_newton_schulz.py (low rank)."""
    from test_gpu_newton_schulz import DT, QUINTIC, definition, rel
    gen = torch.Generator(device="cuda").manual_seed(2)
    for rows, cols in ((72, 136), (136, 72)):
        U = torch.linalg.qr(torch.randn(rows, 3, generator=gen, device="cuda"))[0]
        V = torch.linalg.qr(torch.randn(cols, 3, generator=gen, device="cuda"))[0]
        G = (U @ V.mT).to(DT[dtype])
        O = torch.empty_like(G)
        co = [first, QUINTIC]
        ws = fpo.orthogonalize_grouped([G], [O], steps=2, coeffs=co)
        assert fpo.get_device_status(ws) == fpo.OK
        assert rel(O, definition(G, 2, co)) < (4.5e-3 if dtype == "bf16" else 2e-4)
