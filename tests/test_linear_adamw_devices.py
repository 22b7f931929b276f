"""Every tensor of linear, linear_vjp, adamw_grouped and adamw_state_values is looked at for its device,
the workspace of the caller's and the scales of 8-bit moments among them (no GPU needed: stand-in
tensors and library).  The kernels write the workspace, and the memory of another device may not be
mapped where they run."""
import pytest
import torch

BF, F32 = torch.bfloat16, torch.float32


class _Far(torch.Tensor):
    def get_device(self):
        return 1


class _Near(torch.Tensor):
    def get_device(self):
        return 0


class _Lib:
    """Answers size queries; records what would be launched."""

    def __init__(self):
        self.launched = []

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *a: 4096
        return lambda *a: self.launched.append(name) or 0


@pytest.fixture
def fpo(monkeypatch):
    import paper_2608_14563_gb300 as fpo
    monkeypatch.setattr(fpo, "_current_device", lambda: 0)
    monkeypatch.setattr(fpo, "_stream", lambda s: None)
    monkeypatch.setattr(fpo, "_lib", _Lib())
    monkeypatch.setattr(fpo, "_ptr", lambda t: None if t is None else t.data_ptr())
    return fpo


def _z(*shape, t=BF):
    return torch.zeros(*shape, dtype=t).as_subclass(_Near)


def _ws():
    return _z(8192, t=torch.uint8)


def _calls(fpo):
    """name: (entry point, arguments that are tensors, lists of one or values)."""
    step = fpo.optimizer_desc(clip=fpo.CLIP_STEP)
    n = 300
    return {
        "linear": (fpo.linear, dict(x=_z(4, 16), W=_z(24, 16), y=_z(4, 24), bias=_z(24), residual=_z(4, 24),
                                    z_out=_z(4, 24), workspace=_ws())),
        "linear_vjp": (fpo.linear_vjp, dict(dy=_z(4, 24), x=_z(4, 16), W=_z(24, 16), dx=_z(4, 16), z=_z(4, 24),
                                            z_in=_z(4, 16), dW=_z(24, 16), dbias=_z(24, t=F32),
                                            workspace=_ws())),
        "adamw": (fpo.adamw_grouped, dict(Gs=[_z(n)], opt=step, W_masters=[_z(n, t=F32)],
                                          states1=[_z(n, t=F32)], states2=[_z(n, t=F32)], W_outs=[_z(n)],
                                          workspace=_ws())),
        "adamw, 8-bit moments": (fpo.adamw_grouped, dict(
            Gs=[_z(n)], opt=step, W_masters=[_z(n, t=F32)], states1=[_z(n, t=torch.float8_e4m3fn)],
            states2=[_z(n, t=torch.uint8)], scales1=[_z(2, t=F32)], scales2=[_z(2, t=F32)], W_outs=[_z(n)],
            workspace=_ws())),
        "state values": (fpo.adamw_state_values, dict(codes=_z(n, t=torch.uint8), scales=_z(2, t=F32),
                                                      out=_z(n))),
    }


@pytest.mark.parametrize("name", ["linear", "linear_vjp", "adamw", "adamw, 8-bit moments", "state values"])
def test_each_tensor_of_another_device_is_refused(fpo, name):
    fn, args = _calls(fpo)[name]
    fn(**args)
    assert len(fpo._lib.launched) == 1
    for key, value in args.items():
        if key == "opt":
            continue
        one = value[0] if isinstance(value, list) else value
        far = one.as_subclass(_Far)
        with pytest.raises(ValueError, match="cuda:1"):
            fn(**dict(args, **{key: [far] if isinstance(value, list) else far}))
        assert len(fpo._lib.launched) == 1, key
