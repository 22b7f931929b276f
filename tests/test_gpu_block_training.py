"""A training step of an MLP block of the LayerNorm families as the library's calls make it:
LayerNorm, up-projection with its activation, down-projection onto the residual stream, the way back
through both and the norm, and AdamW over all six tensors; against autograd of the same block in
64 bits.

Tolerances.  fp32: every gradient is a sum of at most T or d_ff products behind four more layers of
roundings, each within 2^-24 of its terms: 2^-24 (T + d_ff + 64) of the tensor's norm.  bf16: eight
tensors are rounded on the way (h, z, a, y, the signals, W's copy), each 2^-8 of its value at most and
independent: sqrt(8) 2^-8 of the norm, twice that as a limit."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rel(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


class Block:
    """The tensors of one block and its calls, in one order on one stream."""

    NAMES = ("W1", "b1", "W2", "b2", "gamma", "beta")

    def __init__(self, fpo, dtype, T, d, f, bits, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.fpo, self.dt, self.T, self.d, self.f = fpo, DT[dtype], T, d, f
        master = dict(W1=rn(f, d) / math.sqrt(d), b1=0.1 * rn(f), W2=rn(d, f) / math.sqrt(f), b2=0.1 * rn(d),
                      gamma=1 + 0.1 * rn(d), beta=0.1 * rn(d))
        self.w = {k: v.to(self.dt) for k, v in master.items()}
        self.master = {k: v.float() for k, v in self.w.items()}
        self.x, self.up = rn(T, d).to(self.dt), (rn(T, d) / T).to(self.dt)
        e = lambda *s, t=None: torch.empty(*s, device="cuda", dtype=t or self.dt)  # noqa: E731
        f32 = torch.float32
        self.h, self.z, self.a, self.y = e(T, d), e(T, f), e(T, f), e(T, d)
        self.dz, self.dh, self.dx = e(T, f), e(T, d), e(T, d)
        self.grads = dict(W1=e(f, d), b1=e(f, t=f32), W2=e(d, f), b2=e(d, t=f32), gamma=e(d, t=f32),
                          beta=e(d, t=f32))
        small = bits == 8
        n = {k: v.numel() for k, v in master.items()}
        self.m = {k: torch.zeros(n[k], device="cuda", dtype=torch.float8_e4m3fn if small else f32) for k in n}
        self.v = {k: torch.zeros(n[k], device="cuda", dtype=torch.uint8 if small else f32) for k in n}
        self.sc = [{k: torch.zeros(-(-n[k] // 256), device="cuda") for k in n} if small else None
                   for _ in range(2)]

    def forward(self, act):
        fpo, w = self.fpo, self.w
        fpo.layernorm(self.x, w["gamma"], w["beta"], self.h)
        fpo.linear(self.h, w["W1"], self.a, bias=w["b1"], act=act, z_out=self.z)
        fpo.linear(self.a, w["W2"], self.y, bias=w["b2"], residual=self.x)

    def backward(self, act):
        fpo, w, g = self.fpo, self.w, self.grads
        fpo.linear_vjp(self.up, self.a, w["W2"], self.dz, act_in=act, z_in=self.z, dW=g["W2"], dbias=g["b2"])
        fpo.linear_vjp(self.dz, self.h, w["W1"], self.dh, dW=g["W1"], dbias=g["b1"])
        fpo.layernorm_vjp(self.dh, self.x, w["gamma"], self.dx, min_rms=0.0, dgamma=g["gamma"],
                          dbeta=g["beta"])

    def step(self, t):
        opt = self.fpo.optimizer_desc(self.fpo.OPT_ADAMW, lr=1e-2, step=t, clip=self.fpo.CLIP_STEP)
        k, cut = self.NAMES, lambda d: None if d is None else [d[n] for n in self.NAMES]  # noqa: E731
        self.fpo.adamw_grouped(cut(self.grads), opt, cut(self.master), cut(self.m), cut(self.v),
                               scales1=cut(self.sc[0]), scales2=cut(self.sc[1]), W_outs=cut(self.w),
                               weight_decays=[0.1 if n[0] == "W" else 0.0 for n in k], seed=11)

    def train(self, act, t):
        self.forward(act)
        self.backward(act)
        self.step(t)


def reference(b, name):
    """y, dx and the gradients of <up, y> in 64 bits."""
    t = {k: v.double().requires_grad_() for k, v in {**b.w, "x": b.x}.items()}
    F = torch.nn.functional
    h = F.layer_norm(t["x"], (b.d,), t["gamma"], t["beta"], 1e-5)
    z = F.linear(h, t["W1"], t["b1"])
    a = {"gelu": F.gelu, "gelu_tanh": lambda z: F.gelu(z, approximate="tanh"), "silu": F.silu}[name](z)
    y = F.linear(a, t["W2"], t["b2"]) + t["x"]
    (b.up.double() * (y - t["x"])).sum().backward()  # (the residual's own gradient is up)
    return y.detach(), {k: v.grad for k, v in t.items()}


CASES = [("f32", 37, 40, 120, "gelu"), ("f32", 300, 65, 129, "silu"), ("bf16", 3, 64, 256, "gelu_tanh"),
         ("bf16", 200, 256, 384, "gelu"), ("bf16", 700, 264, 1032, "silu")]


@pytest.mark.parametrize("dtype,T,d,f,name", CASES)
def test_gradients_of_a_block(fpo, dtype, T, d, f, name):
    b = Block(fpo, dtype, T, d, f, 32)
    act = {"gelu": fpo.ACT_GELU, "gelu_tanh": fpo.ACT_GELU_TANH, "silu": fpo.ACT_SILU}[name]
    b.forward(act)
    b.backward(act)
    y, grads = reference(b, name)
    lim = 2.0 ** -24 * (T + f + 64) if dtype == "f32" else 2 * math.sqrt(8) * 2.0 ** -8
    assert rel(b.y, y) <= lim
    for k in Block.NAMES:
        assert rel(b.grads[k], grads[k]) <= lim, k
    assert rel(b.dx, grads["x"]) <= lim


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_trains_as_the_eager_one(fpo, bits):
    """Three steps: eager, and one captured step replayed while the eager block's memory lives."""
    make = lambda: Block(fpo, "bf16", 200, 256, 384, bits, seed=3)  # noqa: E731
    act = fpo.ACT_GELU_TANH
    eager, graphed = make(), make()
    before = eager.master["W1"].clone()
    for _ in range(3):
        eager.train(act, 5)
    graphed.train(act, 5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.train(act, 5)
    graph.replay()
    graph.replay()
    assert not torch.equal(eager.master["W1"], before)
    for k in Block.NAMES:
        assert torch.equal(eager.master[k], graphed.master[k]) and torch.equal(eager.w[k], graphed.w[k])
        assert torch.equal(eager.m[k].view(torch.uint8), graphed.m[k].view(torch.uint8))
        assert torch.equal(eager.v[k].view(torch.uint8), graphed.v[k].view(torch.uint8))
    assert torch.equal(eager.y, graphed.y)


def test_activations_feed_the_pseudogradient(fpo):
    """The up-projection's output as a cached activation of the layer update: the same G as dW."""
    b = Block(fpo, "bf16", 200, 256, 384, 32)
    b.forward(fpo.ACT_GELU)
    b.backward(fpo.ACT_GELU)
    G = torch.empty(256, 384, dtype=torch.bfloat16, device="cuda")
    fpo.layer_update(b.up, b.a, 0.0, G_out=G)
    want = b.up.double().t() @ b.a.double()
    assert rel(G, want) <= 2.0 ** -8 and rel(b.grads["W2"], want) <= 2.0 ** -8
