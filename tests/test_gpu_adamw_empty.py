"""Empty tensors among those of fpo_adamw_grouped: the others get the bits that they get without them."""
import pytest
import torch

from test_gpu_adamw import Tensors

pytestmark = pytest.mark.gpu

SIZES = [0, 300, 0, 0, 5, 0, 4097]


def _pick(x, keep):
    y = Tensors.__new__(Tensors)
    y.n, y.bits = [x.n[k] for k in keep], x.bits
    for name in ("G", "W", "out", "m", "v", "ms", "vs", "decay"):
        ts = getattr(x, name)
        setattr(y, name, None if ts is None else
                [t.clone() if isinstance(t, torch.Tensor) else t for t in (ts[k] for k in keep)])
    return y


def _same(a, b):
    return a is b or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("clip", [0, 1, 2])
def test_fp32_moments_as_in_a_call_of_the_others(fpo, clip):
    x = Tensors(SIZES, 32)
    keep = [k for k, n in enumerate(SIZES) if n]
    alone, start = _pick(x, keep), _pick(x, keep)
    for t in (1, 2):
        x.step(fpo, t, clip)
        alone.step(fpo, t, clip)
    for i, k in enumerate(keep):
        for name in ("W", "m", "v", "out"):
            assert _same(getattr(x, name)[k], getattr(alone, name)[i]), (name, k)
        assert not torch.equal(x.W[k], start.W[i])


@pytest.mark.parametrize("clip", [0, 1, 2])
def test_8_bit_moments_as_beside_others(fpo, clip):
    """(Their rounding depends on a tensor's place: the empty ones' places are taken by others.)"""
    x = Tensors(SIZES, 8)
    other = Tensors([n or 9 for n in SIZES], 8)
    keep = [k for k, n in enumerate(SIZES) if n]
    for k in keep:
        for name in ("G", "W", "out"):
            t = getattr(x, name)[k]
            getattr(other, name)[k] = None if t is None else t.clone()
    start = [w.clone() for w in x.W]
    for t in (1, 2):
        x.step(fpo, t, clip)
        other.step(fpo, t, clip)
    for k in keep:
        for name in ("W", "m", "v", "ms", "vs", "out"):
            assert _same(getattr(x, name)[k], getattr(other, name)[k]), (name, k)
        assert not torch.equal(x.W[k], start[k])
