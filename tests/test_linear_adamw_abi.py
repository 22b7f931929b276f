"""fpo_linear, fpo_linear_vjp and fpo_adamw_grouped refuse bad arguments on the host, and say how
much workspace they need (no GPU needed)."""
import ctypes

import pytest
import torch

from test_binding_streams import _Stream, world  # noqa: F401  (a fixture)

OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, ARCH, CUDA, ARG = 0, 1, 2, 3, 4, 5, 6, 7, 10
NO_GPU = (ARCH, CUDA)  # every argument is in order: the device is what is missing
P = 1 << 24            # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def fpo():
    import paper_2608_14563_gb300 as fpo
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where no call gets as far as a launch")
    return fpo


def test_linear_refusals(fpo):
    need = fpo.linear_workspace(300, 512, 264)
    assert need >= 256

    def call(T=300, n=512, k=264, dtype=1, act=2, x=P, w=2 * P, b=3 * P, r=4 * P, y=5 * P, z=6 * P,
             ws=8 * P, size=None):
        size = fpo.linear_workspace(T, n, k, dtype) if size is None else size
        return fpo._lib.fpo_linear(T, n, k, dtype, act, x, w, b, r, y, z, ws, size, None)

    assert call() in NO_GPU and call(b=None, r=None, z=None) in NO_GPU and call(r=5 * P) in NO_GPU
    assert call(dtype=2) == DTYPE and call(dtype=-1) == DTYPE
    assert call(T=-1) == SHAPE and call(n=0) == SHAPE and call(k=0) == SHAPE
    assert call(n=516) == SHAPE and call(k=260) == SHAPE and call(T=1 << 31) == SHAPE
    big = (1 << 30) + 8
    assert call(T=big, size=1 << 40) == SHAPE and call(n=big) == SHAPE and call(k=big, dtype=0) == SHAPE
    assert call(n=515, k=3, dtype=0, size=256) in NO_GPU
    assert call(act=5) == ARG and call(act=-1) == ARG
    assert call(x=None) == NULL and call(w=None) == NULL and call(y=None) == NULL
    for name in "xwbryz":
        assert call(**{name: 7 * P + 8}) == ALIGN
    assert call(ws=None) == WORKSPACE and call(size=need - 1) == WORKSPACE
    assert call(ws=8 * P + 16) == ALIGN
    # outputs over inputs, each other, the workspace; whole and in parts
    assert call(y=P) == ARG and call(z=5 * P) == ARG and call(y=2 * P + 512) == ARG
    assert call(r=5 * P + 16) == ARG and call(b=5 * P + 32) == ARG and call(ws=P) == ARG
    assert call(z=4 * P) == ARG
    # inputs may share memory
    assert call(x=2 * P) in NO_GPU
    # nothing to read or write without tokens
    assert call(T=0, x=None, w=None, y=None, b=None, r=None, z=None) in NO_GPU


def test_linear_vjp_refusals(fpo):
    need = fpo.linear_vjp_workspace(300, 512, 264, 1, 2)
    assert need >= 300 * 512 * 2

    def call(T=300, n=512, k=264, dtype=1, act=2, dy=P, z=2 * P, x=3 * P, w=4 * P, act_in=4, zi=5 * P,
             dx=6 * P, dw=7 * P, db=9 * P, ws=16 * P, size=None):
        size = fpo.linear_vjp_workspace(T, n, k, dtype, act) if size is None else size
        return fpo._lib.fpo_linear_vjp(T, n, k, dtype, act, dy, z, x, w, act_in, zi, dx, dw, db, ws, size,
                                       None)

    assert call() in NO_GPU
    assert call(dtype=3) == DTYPE and call(T=-1) == SHAPE and call(n=4) == SHAPE and call(k=4) == SHAPE
    assert call(act=9, size=1 << 30) == ARG and call(act_in=-1) == ARG
    assert call(dx=None, dw=None, db=None) == NULL
    for name in ("dy", "z", "x", "w", "zi"):
        assert call(**{name: None}) == NULL
    # what is not read may be missing
    assert call(act=0, z=None) in NO_GPU and call(act_in=0, zi=None) in NO_GPU
    assert call(dx=None, w=None, zi=None) in NO_GPU and call(dw=None, x=None) in NO_GPU
    assert call(dx=None, dw=None, w=None, x=None, zi=None) in NO_GPU
    for name in ("dy", "z", "x", "w", "zi", "dx", "dw", "db"):
        assert call(**{name: 10 * P + 8}) == ALIGN
    assert call(ws=None) == WORKSPACE and call(size=need - 1) == WORKSPACE
    assert call(ws=16 * P + 64) == ALIGN
    for out, inp in (("dx", P), ("dx", 5 * P), ("dw", 4 * P), ("dw", 6 * P + 16)):
        assert call(**{out: inp}) == ARG, (out, inp)
    assert call(db=7 * P) == ARG and call(ws=6 * P) == ARG
    assert call(T=0, dy=None, z=None, x=None, w=None, zi=None) in NO_GPU


def test_workspaces_are_what_the_header_says(fpo):
    for T, n, k in ((1, 8, 8), (4, 11008, 4096), (5, 264, 4096), (16, 4096, 11008), (17, 256, 384), (32, 16384, 512),
                    (33, 4096, 11008),
                    (129, 256, 4096), (200, 384, 256), (4096, 4096, 11008), (16384, 11008, 4096)):
        extra = fpo.linear_workspace(T, n, k) - 256
        padded = next((p for p in (16, 32) if T <= p), None)
        if T <= 4:
            assert extra == 0
        elif padded:
            counters = -(-(-(-n // 128) * 16) // 256) * 256
            assert 0 < extra - counters <= 2 * 152 * 512 * padded
        else:
            assert 0 <= extra <= 3 * 76 * 256 * 256 * 4
        assert fpo.linear_workspace(T, n, k, fpo.F32) == 256
        for act in (fpo.ACT_NONE, fpo.ACT_SILU):
            v = fpo.linear_vjp_workspace(T, n, k, fpo.BF16, act)
            parts = 4 * n if T > (2048 if act else 8192) else 0  # below that the ranges are a cluster
            assert v - (T * n * 2 if act else 0) >= 256 + parts
    assert fpo.linear_workspace(0, 64, 64) == 256 and fpo.linear_vjp_workspace(0, 64, 64) == 256
    assert fpo.linear_workspace(4, 12, 64) == 0 and fpo.linear_workspace(-1, 64, 64) == 0
    assert fpo.linear_vjp_workspace(4, 64, 64, 7) == 0 and fpo.linear_vjp_workspace(4, 64, 64, 1, 9) == 0
    assert fpo.adamw_workspace([1000, 5]) == 0
    assert fpo.adamw_workspace([4096 * 11008, 5], fpo.CLIP_STEP) <= 4096 * 11008 // 256 + 4096
    assert fpo.adamw_workspace([-1], fpo.CLIP_STEP) == 0


def _tensors(fpo, *specs):
    """Tensors of 300 elements at made-up addresses, `specs`: dicts of changed fields."""
    t = (fpo.AdamwTensor * len(specs))()
    for k, spec in enumerate(specs):
        base = P * 16 * (k + 1)
        fields = dict(n=300, G=base, W_master=base + P, W_out=base + 2 * P, state1=base + 3 * P,
                      state2=base + 4 * P, scale1=base + 5 * P, scale2=base + 6 * P, g_dtype=1, w_dtype=1,
                      state_bits=8, weight_decay=0.1)
        fields.update(spec)
        for name, v in fields.items():
            setattr(t[k], name, v)
    return t


def test_adamw_refusals(fpo):
    def call(*specs, n=None, ws=None, size=0, **opt):
        t = _tensors(fpo, *specs)
        o = fpo.AdamwDesc(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, clip_frac=0.01, step=1,
                                    clip=fpo.CLIP_NONE), **opt})
        return fpo._lib.fpo_adamw_grouped(len(specs) if n is None else n, t, ctypes.byref(o), 7, ws, size,
                                          None)

    base = 16 * P
    assert call({}) in NO_GPU and call({}, {}, {"state_bits": 32}) in NO_GPU
    assert call({}, n=0) == SHAPE and call({}, n=-3) == SHAPE
    assert call({"n": -1}) == SHAPE and call({"n": (1 << 40) + 1}) == SHAPE
    assert call({"g_dtype": 2}) == DTYPE and call({"w_dtype": -1}) == DTYPE
    assert call({"state_bits": 16}) == ARG and call({"weight_decay": float("nan")}) == ARG
    assert call({}, eps=float("nan")) == ARG and call({}, eps=-1e-8) == ARG
    assert call({}, step=0) == ARG and call({}, beta1=1.0) == ARG and call({}, beta2=-0.1) == ARG
    assert call({}, lr=float("nan")) == ARG and call({}, clip=3) == ARG
    assert call({}, clip_frac=-1.0) == ARG
    for name in ("G", "W_master", "state1", "state2", "scale1", "scale2"):
        assert call({name: None}) == NULL
    assert call({"W_out": None}) in NO_GPU and call({"state_bits": 32, "scale1": None}) in NO_GPU
    for name in ("G", "W_master", "W_out", "state1", "state2"):
        assert call({name: base + 9 * P + 8}) == ALIGN
    assert call({"scale1": base + 9 * P + 2}) == ALIGN and call({"scale2": base + 9 * P + 4}) in NO_GPU
    # empty tensors are skipped
    assert call({"n": 0, "G": None, "W_master": None, "state1": None, "state2": None, "scale1": None,
                 "scale2": None}, {}) in NO_GPU
    # memory used twice
    assert call({"W_out": base + P}) == ARG  # bf16 over the fp32 master
    assert call({"W_out": base + P, "w_dtype": 0}) in NO_GPU
    assert call({"state2": base + 3 * P}) == ARG and call({"G": base + P}) == ARG
    assert call({}, {"W_master": base + P}) == ARG and call({}, {"state1": base + 3 * P + 16}) == ARG
    assert call({"scale1": base + 3 * P + 4}) == ARG
    assert call({}, {"G": base}) in NO_GPU  # a shared gradient
    # the clip's workspace
    clip = dict(clip=fpo.CLIP_STEP)
    need = fpo.adamw_workspace([300, 300], fpo.CLIP_STEP)
    assert need > 0
    assert call({}, {}, **clip) == WORKSPACE
    assert call({}, {}, ws=P, size=need - 1, **clip) == WORKSPACE
    assert call({}, {}, ws=P + 16, size=need, **clip) == ALIGN
    assert call({}, {}, ws=base, size=need, **clip) == ARG
    assert call({}, {}, ws=P, size=need, **clip) in NO_GPU
    lib = fpo._lib
    assert lib.fpo_adamw_grouped(1, None, ctypes.byref(fpo.AdamwDesc()), 0, None, 0, None) == NULL
    assert lib.fpo_adamw_grouped(1, _tensors(fpo, {}), None, 0, None, 0, None) == NULL


def test_state_values_refusals(fpo):
    def call(n=300, moment=1, codes=P, scales=2 * P, dtype=1, out=3 * P):
        return fpo._lib.fpo_adamw_state_values(n, moment, codes, scales, dtype, out, None)

    assert call() in NO_GPU and call(n=0, codes=None, scales=None, out=None) in NO_GPU
    assert call(moment=0) == ARG and call(moment=3) == ARG and call(dtype=5) == DTYPE
    assert call(n=-1) == SHAPE and call(codes=None) == NULL and call(scales=None) == NULL
    assert call(out=None) == NULL and call(codes=P + 4) == ALIGN and call(out=P + 8) == ALIGN
    assert call(scales=P + 1) == ALIGN and call(out=P) == ARG and call(out=2 * P) == ARG


def test_binding_checks_shapes_and_types(fpo):
    """What the C entry points cannot see: shapes and types of the tensors behind the pointers."""
    bf, f32 = torch.bfloat16, torch.float32
    z = lambda *s, t=bf: torch.zeros(*s, dtype=t)  # noqa: E731
    x, W, y = z(4, 16), z(24, 16), z(4, 24)
    for bad in (dict(x=z(4, 8)), dict(y=z(4, 16)), dict(y=z(4, 24, t=f32)), dict(bias=z(16)),
                dict(bias=z(24, t=f32)), dict(residual=z(1, 24)), dict(z_out=z(24, 4))):
        a = dict(x=x, W=W, y=y, **{})
        a.update(bad)
        with pytest.raises(ValueError):
            fpo.linear(a.pop("x"), a.pop("W"), a.pop("y"), **a)
    with pytest.raises(ValueError, match="CUDA"):
        fpo.linear(x, W, y)
    dy, dx = z(4, 24), z(4, 16)
    for bad in (dict(x=z(3, 16)), dict(dx=z(4, 24)), dict(dW=z(16, 24)), dict(dbias=z(24)),
                dict(z=z(4, 16)), dict(z_in=z(4, 24)), dict(W=z(24, 8))):
        a = dict(dy=dy, x=x, W=W, dx=dx)
        a.update(bad)
        with pytest.raises(ValueError):
            fpo.linear_vjp(a.pop("dy"), a.pop("x"), a.pop("W"), a.pop("dx"), **a)
    opt = fpo.optimizer_desc(clip=fpo.CLIP_NONE)
    n = 300
    G, Wm, m, v = z(n), z(n, t=f32), z(n, t=f32), z(n, t=f32)
    m8, v8, sc = torch.zeros(n, dtype=torch.float8_e4m3fn), z(n, t=torch.uint8), z(2, t=f32)
    with pytest.raises(ValueError):
        fpo.adamw_grouped([], opt, [], [], [])
    for args, kw in ((([G], opt, [Wm, Wm], [m], [v]), {}), (([G], opt, [z(n)], [m], [v]), {}),
                     (([G], opt, [z(20, t=f32)], [m], [v]), {}), (([G], opt, [Wm], [m], [v8]), {}),
                     (([G], opt, [Wm], [m8], [v]), {}), (([G], opt, [Wm], [m8], [v8]), {}),
                     (([G], opt, [Wm], [m8], [v8]), dict(scales1=[sc], scales2=[None])),
                     (([G], opt, [Wm], [m8], [v8]), dict(scales1=[sc], scales2=[z(3, t=f32)])),
                     (([G], opt, [Wm], [m], [v]), dict(W_outs=[z(20)])),
                     (([G], opt, [Wm], [m], [v]), dict(weight_decays=[0.1, 0.2])),
                     (([G], fpo.optimizer_desc(fpo.OPT_SGD), [Wm], [m], [v]), {})):
        with pytest.raises(ValueError):
            fpo.adamw_grouped(*args, **kw)
    with pytest.raises(TypeError):
        fpo.adamw_grouped([z(n, t=torch.float16)], opt, [Wm], [m], [v])
    with pytest.raises(TypeError):
        fpo.adamw_state_values(m, sc, z(n))
    with pytest.raises(ValueError):
        fpo.adamw_state_values(v8, sc, z(20))
    with pytest.raises(ValueError):
        fpo.adamw_state_values(v8, z(1, t=f32), z(n))


class _Far(torch.Tensor):
    def get_device(self):
        return 1


def test_any_tensor_of_another_device_is_refused(fpo, monkeypatch):
    """The memory of another device may not be mapped where the kernels run (stand-in tensors)."""
    monkeypatch.setattr(fpo, "_current_device", lambda: 0)
    monkeypatch.setattr(fpo, "_ptr", lambda t: None if t is None else t.data_ptr())
    bf, f32 = torch.bfloat16, torch.float32
    z = lambda *s, t=bf: torch.zeros(*s, dtype=t)  # noqa: E731
    opt = fpo.optimizer_desc(clip=fpo.CLIP_NONE)
    calls = [
        (fpo.linear, dict(x=z(4, 16), W=z(24, 16), y=z(4, 24), bias=z(24), residual=z(4, 24), z_out=z(4, 24))),
        (fpo.linear_vjp, dict(dy=z(4, 24), x=z(4, 16), W=z(24, 16), dx=z(4, 16), z=z(4, 24), z_in=z(4, 16),
                              dW=z(24, 16), dbias=z(24, t=f32))),
        (fpo.adamw_state_values, dict(codes=z(300, t=torch.uint8), scales=z(2, t=f32), out=z(300)))]
    for fn, args in calls:
        for name in args:
            far = dict(args, **{name: args[name].as_subclass(_Far)})
            with pytest.raises(ValueError, match="cuda:1"):
                fn(**far)
    lists = dict(Gs=[z(300)], W_masters=[z(300, t=f32)], states1=[z(300, t=f32)], states2=[z(300, t=f32)],
                 W_outs=[z(300)])
    for name in lists:
        far = dict(lists, **{name: [lists[name][0].as_subclass(_Far)]})
        with pytest.raises(ValueError, match="cuda:1"):
            fpo.adamw_grouped(opt=opt, **far)


def test_rates_reach_the_library_in_double(fpo, monkeypatch):
    seen = []

    class Lib:
        def fpo_adamw_grouped(self, n, table, desc, *rest):
            d = desc._obj
            seen.append((d.lr, d.beta1, d.beta2, d.eps, d.step, d.clip, table[0].weight_decay))
            return 0

    monkeypatch.setattr(fpo, "_lib", Lib())
    monkeypatch.setattr(fpo, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(fpo, "_stream", lambda s: None)
    monkeypatch.setattr(fpo, "_current_device", lambda: 0)
    z = [torch.zeros(8) for _ in range(4)]
    opt = fpo.optimizer_desc(lr=3e-4, beta2=0.999, clip=0, step=5)
    fpo.adamw_grouped(z[:1], opt, z[1:2], z[2:3], z[3:])
    assert seen[-1] == (3e-4, 0.9, 0.999, 1e-8, 5, 0, ctypes.c_float(0.01).value)
    opt.lr, opt.step = 0.125, 6  # a schedule sets the fields
    fpo.adamw_grouped(z[:1], opt, z[1:2], z[2:3], z[3:])
    assert seen[-1] == (0.125, 0.9, 0.999, 1e-8, 6, 0, ctypes.c_float(0.01).value)


@pytest.mark.parametrize("side", [False, True])
def test_memory_belongs_to_the_stream_of_the_call(world, monkeypatch, side):  # noqa: F811
    """A workspace that the binding allocates is the call's stream's."""
    fpo = world.fpo
    monkeypatch.setattr(fpo, "_current_device", lambda: 0)
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)  # noqa: E731
    x, W, y, f = z(4, 16), z(24, 16), z(4, 24), z(300, t=torch.float32)
    for call in (lambda s: fpo.linear(x, W, y, stream=s), lambda s: fpo.linear_vjp(y, x, W, x.clone(), stream=s),
                 lambda s: fpo.adamw_grouped([f], fpo.optimizer_desc(), [f], [f], [f], stream=s)):
        world.allocated.clear()
        call(_Stream(0x20) if side else None)
        assert [s.cuda_stream for _, s in world.allocated] == [0x20 if side else 0x10]
