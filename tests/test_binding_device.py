"""A call whose tensors lie on another device than the current one is refused before anything is
launched (no GPU needed: a stand-in tensor and library)."""
import types

import pytest
import torch

import test_binding_streams as streams


class _Far(torch.Tensor):
    def get_device(self):
        return 1


class _Lib:
    """Answers size queries; nothing may get as far as a launch."""

    def __getattr__(self, name):
        def launch(*args):
            raise AssertionError(name + " was called")
        return (lambda *a: 4096) if name.endswith("_workspace") else launch


@pytest.fixture
def fpo(monkeypatch):
    import paper_2608_14563_gb300 as fpo
    monkeypatch.setattr(fpo, "_current_device", lambda: 0)
    monkeypatch.setattr(fpo, "_lib", _Lib())
    monkeypatch.setattr(fpo, "_ptr", lambda t: None if t is None else t.data_ptr())
    return fpo


def _far(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_Far)


def test_tensors_of_another_device_are_refused(fpo, monkeypatch):
    monkeypatch.setattr(streams, "_z", _far)
    calls = streams._calls(fpo)
    x, w = _far(8, 16), _far(16)
    calls["layernorm"] = lambda s: fpo.layernorm(x, w, w, x.clone(), stream=s)
    calls["rmsnorm_vjp"] = lambda s: fpo.rmsnorm_vjp(x, x, w, x, stream=s)
    calls["layer_signals"] = lambda s: fpo.layer_signals(x, [x], m=[x], gamma_post=[w], stream=s)
    calls["h2d_copy"] = lambda s: fpo.h2d_copy([x], [torch.zeros(8, 16, dtype=torch.bfloat16)], stream=s)
    for name, call in calls.items():
        with pytest.raises(ValueError, match="cuda:1"):
            call(None)


def test_the_current_device_and_host_tensors(fpo):
    fpo._on_current_device(torch.zeros(2))  # refused later, as no CUDA tensor
    near = types.SimpleNamespace(get_device=lambda: 0)
    fpo._on_current_device(near)
