"""Every entry point of the binding that takes a workspace and a stream, whatever kind of callable it is,
is among the calls whose allocations are followed to their stream (no GPU needed)."""
import inspect
import types

import pytest
import torch

import test_binding_streams as streams
from test_binding_streams import _Stream, world  # noqa: F401  (a fixture)

# (these read a workspace that they are given)
GIVEN = {"get_device_status", "direct_fixup_rows"}


def _entries(fpo):
    found = set()
    for name, f in vars(fpo).items():
        if not callable(f) or inspect.isclass(f):
            continue
        try:
            names = set(inspect.signature(f).parameters)
        except (TypeError, ValueError):  # a builtin without a signature
            continue
        if {"workspace", "stream"} <= names:
            found.add(name)
    return found


def _calls(fpo):
    """The entry points that are not plain functions."""
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)  # noqa: E731
    x, W, y, f = z(4, 16), z(24, 16), z(4, 24), z(300, t=torch.float32)
    m, v, sc = z(300, t=torch.float8_e4m3fn), z(300, t=torch.uint8), z(2, t=torch.float32)
    clip = fpo.optimizer_desc()
    return {
        "linear": [lambda s: fpo.linear(x, W, y, stream=s)],
        "linear_vjp": [lambda s: fpo.linear_vjp(y, x, W, x.clone(), stream=s),
                       lambda s: fpo.linear_vjp(y, None, None, None, dbias=z(24, t=torch.float32), stream=s)],
        "adamw_grouped": [lambda s: fpo.adamw_grouped([f], clip, [f], [f], [f], stream=s),
                          lambda s: fpo.adamw_grouped([f], clip, [f], [m], [v], scales1=[sc], scales2=[sc],
                                                      stream=s)],
    }


def test_every_entry_point_with_a_workspace_is_followed(world):  # noqa: F811
    functions, others = set(streams._calls(world.fpo)), set(_calls(world.fpo))
    assert not functions & others
    assert _entries(world.fpo) - GIVEN == functions | others


def test_a_callable_object_is_seen(world, monkeypatch):  # noqa: F811
    def extra(x, *, workspace=None, stream=None):
        pass

    for entry in (extra, world.fpo._entry(extra)):
        monkeypatch.setattr(world.fpo, "extra", entry, raising=False)
        assert "extra" in _entries(world.fpo)
    assert "extra" not in dict(inspect.getmembers(world.fpo, inspect.isfunction))


@pytest.mark.parametrize("kind", ["current", "torch stream", "other handle"])
def test_their_memory_belongs_to_the_stream_of_the_call(world, monkeypatch, kind):  # noqa: F811
    monkeypatch.setattr(world.fpo, "_current_device", lambda: 0)
    stream = {"current": None, "torch stream": _Stream(0x20),
              "other handle": types.SimpleNamespace(cuda_stream=0x20)}[kind]
    for name, calls in _calls(world.fpo).items():
        for call in calls:
            world.allocated.clear()
            world.recorded.clear()
            call(stream)
            assert [s.cuda_stream for _, s in world.allocated] == [0x20 if stream else 0x10], name
            assert not world.recorded, name
