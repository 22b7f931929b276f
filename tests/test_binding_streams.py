"""The memory that the binding allocates for a call belongs to the stream the call runs on (no GPU
needed: a stand-in library and allocator record what happens).

A workspace taken on the current stream while the call is given another one could still be in use
by earlier work of the current stream, and would be handed to its next allocation while the call's
kernels still run."""
import contextlib
import types

import pytest
import torch

T, D, F, V = 4000, 64, 128, 256


class _Lib:
    """Every entry point succeeds, every size query says 4096 bytes."""

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *a: 4096
        return lambda *a: 0


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def world(monkeypatch):
    import paper_2608_14563_gb300 as fpo
    w = types.SimpleNamespace(fpo=fpo, current=[_Stream(0x10)], allocated=[], recorded=[])

    @contextlib.contextmanager
    def use(stream):
        w.current.append(stream)
        yield
        w.current.pop()

    class Tensor(torch.Tensor):
        def record_stream(self, stream):
            w.recorded.append((self, stream))

    real_empty = torch.empty

    def empty(*a, **kw):
        t = real_empty(*a, **kw).as_subclass(Tensor)
        w.allocated.append((t, w.current[-1]))
        return t

    monkeypatch.setattr(fpo, "_lib", _Lib())
    monkeypatch.setattr(fpo, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(fpo, "_raw_stream", lambda dev: w.current[-1].cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: w.current[-1])
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: _Stream(handle))
    monkeypatch.setattr(torch, "empty", empty)
    return w


def _z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def _calls(fpo):
    g, A, W32 = _z(T, D), _z(T, F), _z(D, F, dtype=torch.float32)
    W16, y = _z(D, F), torch.zeros(T, dtype=torch.int32)
    d32 = _z(D, dtype=torch.float32)
    opt, muon = fpo.optimizer_desc(), fpo.muon_desc()
    return {
        "error_signal": lambda s: fpo.error_signal(g, _z(D), _z(V, D), y, g, stream=s),
        "layer_update": lambda s: fpo.layer_update(g, A, 0.1, W_master=W32, stream=s),
        "layer_update_grouped": lambda s: fpo.layer_update_grouped(g, [A], 0.1, W_masters=[W32],
                                                                   stream=s),
        "layer_update_grouped_signals": lambda s: fpo.layer_update_grouped_signals(
            [g], [A], 0.1, W_masters=[W32], stream=s),
        "layer_optimize_grouped": lambda s: fpo.layer_optimize_grouped([g], [A], opt, [W32], stream=s),
        "orthogonalize_grouped": lambda s: fpo.orthogonalize_grouped([W16], [W16], stream=s),
        "layer_muon_grouped": lambda s: fpo.layer_muon_grouped([g], [A], muon, [W32], [W32.clone()],
                                                               stream=s),
        "gate_up_signals": lambda s: fpo.gate_up_signals(g, W16, A, A, A, A, stream=s),
        "layernorm_vjp": lambda s: fpo.layernorm_vjp(g, g, None, None, dgamma=d32, stream=s),
        "cosine": lambda s: fpo.cosine(W16, W16, stream=s),
        "cosine_grouped": lambda s: fpo.cosine_grouped([W16], [W16], stream=s),
        "layer_grad_cosine_grouped": lambda s: fpo.layer_grad_cosine_grouped(g, [A], [W16], [W16],
                                                                             stream=s),
        "norm_ratio": lambda s: fpo.norm_ratio([W16], [W16], stream=s),
    }


def test_every_call_with_a_workspace_is_here(world):
    import inspect
    names = {n for n, f in inspect.getmembers(world.fpo, inspect.isfunction)
             if {"workspace", "stream"} <= set(inspect.signature(f).parameters)}
    # (these read a workspace that they are given)
    assert names - {"get_device_status", "direct_fixup_rows"} == set(_calls(world.fpo))


@pytest.mark.parametrize("foreign", [False, True], ids=["torch stream", "other handle"])
def test_memory_belongs_to_the_stream_of_the_call(world, foreign):
    for name, call in _calls(world.fpo).items():
        side = types.SimpleNamespace(cuda_stream=0x20) if foreign else _Stream(0x20)
        world.allocated.clear()
        world.recorded.clear()
        call(side)
        made = [(t, s.cuda_stream) for t, s in world.allocated]
        assert made and all(s == 0x20 for _, s in made), name
        # results that the caller reads are not reused before the current stream is past them
        read = [t for t, _ in made if t.dtype == torch.float64]
        assert len(world.recorded) == len(read), name
        assert all(a is b and s is world.current[0]
                   for (a, s), b in zip(world.recorded, read)), name


def test_without_a_stream_the_current_one_is_used(world):
    for name, call in _calls(world.fpo).items():
        world.allocated.clear()
        call(None)
        assert world.allocated and all(s is world.current[0] for _, s in world.allocated), name
        assert not world.recorded, name


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["vjp", "orthogonalize"])
def test_side_stream_calls_leave_the_current_stream_alone(fpo, kind):
    """Calls on a stream that is still busy, without a workspace of the caller's, while the current
    stream allocates and fills tensors of the workspace's size: neither sees the other."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    if kind == "vjp":
        x, g = (torch.randn(700, 264, generator=gen, device="cuda").bfloat16() for _ in range(2))
        need = fpo.layernorm_vjp_workspace(700, 264)
        outs = [[torch.empty(264, device="cuda") for _ in range(2)] for _ in range(2)]

        def call(o, **kw):
            fpo.layernorm_vjp(g, x, None, None, dgamma=o[0], dbeta=o[1], **kw)
    else:
        G = torch.randn(72, 136, generator=gen, device="cuda").bfloat16()
        need = fpo.orthogonalize_workspace(1, 72, 136)
        outs = [[torch.empty_like(G)] for _ in range(2)]

        def call(o, **kw):
            fpo.orthogonalize_grouped([G], o, **kw)

    assert need > 0
    call(outs[0])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)  # some ten milliseconds
    fills = []
    for i in range(8):
        call(outs[1], stream=s)
        fills.append(torch.full((need,), i, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert all((f == i).all() for i, f in enumerate(fills))
