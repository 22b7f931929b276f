"""Measured cases of the linear layer, its backward pass and AdamW over many tensors.

Kinds:

* ``linear``  Y = act(X W^T + b) + R, and the pre-activation where a backward pass will read it
* ``vjp``     its backward pass: the signal for the layer's input (through the activation below
              it where there is one), and the gradients of the weight and the bias
* ``adamw``   one AdamW step over every tensor of some MLP blocks (two matrices, their biases and
              a LayerNorm's weights each), the states in fp32 or in 8 bits

``run`` computes them in elementary torch operations in fp32, or, with ``own`` set, through
the library's entry points.  ``exact`` states the same definitions once more in fp64.

Sizes are those of the repository's workloads and tests, or generic ones of the same ranges.
Inputs: activations X ~ N(0, 1) (after a norm) or act(N) (below an activation), W ~ N(0, 0.02^2),
signals of the size that a mean-reduced cross-entropy leaves, AdamW states as they are after
a hundred steps.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LR, BETA1, BETA2, ADAM_EPS, WEIGHT_DECAY, CLIP_FRAC = 3e-4, 0.9, 0.999, 1e-8, 0.1, 0.01
STEP = 100
BLOCK = 256           # elements that share the scales of their 8-bit states
WORD = 0xffffffff
# odd 32-bit constants of the rounding noise: fractions of the golden ratio, sqrt(2), sqrt(3)
PHI, SQRT2, SQRT3 = 0x9E3779B9, 0x6A09E667, 0xBB67AE85


# ------------------------------------------------------------------------ the cases
def listed():
    return [
        # one token through an up-projection of the 7B shape: the weights' bytes
        dict(name="linear-one-token", kind="linear", dtype="bf16", T=1, d_in=4096, d_out=11008,
             act="gelu_tanh", bias=True, residual=False, keep=False),
        # the unit-test-sized layer with everything in its epilogue, a ragged token count
        dict(name="linear-short", kind="linear", dtype="bf16", T=200, d_in=256, d_out=384,
             act="silu", bias=True, residual=True, keep=True),
        # the training batch of the 7B-shaped workload, up-projection: the pre-activation is kept
        dict(name="linear-up-training", kind="linear", dtype="bf16", T=16384, d_in=4096,
             d_out=11008, act="gelu_tanh", bias=True, residual=False, keep=True),
        # two packed sequences through the down-projection, added to the residual stream
        dict(name="linear-down-residual", kind="linear", dtype="bf16", T=4096, d_in=11008,
             d_out=4096, act="none", bias=True, residual=True, keep=False),
        # an fp32 reference run with odd sizes: rows that are not aligned to 16 bytes
        dict(name="linear-f32-odd", kind="linear", dtype="f32", T=777, d_in=767, d_out=1537,
             act="gelu", bias=True, residual=False, keep=True),
        # the unit-test-sized down-projection, through the activation below it
        dict(name="vjp-short", kind="vjp", dtype="bf16", T=200, d_in=384, d_out=256, act="none",
             act_in="silu", bias=True),
        # four packed sequences through a 7B down-projection, through the activation below it
        dict(name="vjp-down-training", kind="vjp", dtype="bf16", T=8192, d_in=11008, d_out=4096,
             act="none", act_in="gelu_tanh", bias=True),
        # an fp32 reference run of a layer with its own activation, odd sizes
        dict(name="vjp-f32-odd", kind="vjp", dtype="f32", T=513, d_in=511, d_out=1025, act="gelu",
             act_in="none", bias=True),
        # every tensor of eight unit-test-sized blocks: what one launch over many tensors costs
        dict(name="adamw-small-blocks", kind="adamw", bits=32, layers=8, d=256, d_ff=384,
             clip="none"),
        # odd-sized blocks with 8-bit states: blocks of 256 elements that end inside a row
        dict(name="adamw8-odd", kind="adamw", bits=8, layers=3, d=333, d_ff=1001, clip="none"),
        # a block of the 7B shape with the relative clip on the step, as the paper trains
        dict(name="adamw-7b-clip", kind="adamw", bits=32, layers=1, d=4096, d_ff=11008,
             clip="step"),
        # two blocks of the 7B shape with 8-bit states
        dict(name="adamw8-7b", kind="adamw", bits=8, layers=2, d=4096, d_ff=11008, clip="none"),
    ]


def _log(rng, lo, hi, mult=1):
    """A size spread over the logarithm of [lo, hi], a multiple of mult."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / mult)) * mult, -(-lo // mult) * mult), hi // mult * mult)


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "vjp", "vjp", "adamw", "adamw"])
    acts = ["none", "relu", "gelu", "gelu_tanh", "silu"]
    while True:
        if kind == "adamw":
            c = dict(kind=kind, bits=rng.choice([8, 8, 32]), layers=rng.choice([1, 2, 3, 6]),
                     d=_log(rng, 8, 8192), d_ff=_log(rng, 16, 16384),
                     clip=rng.choice(["none", "none", "step", "gradient"]))
            if work(c)["bytes"] <= 3e9:
                return c
            continue
        dtype = rng.choice(["bf16", "bf16", "f32"])
        mult, hi = (8, 16384) if dtype == "bf16" else (1, 3000)
        c = dict(kind=kind, dtype=dtype, T=_log(rng, 1, 16384), d_in=_log(rng, 8, hi, mult),
                 d_out=_log(rng, 8, hi, mult), act=rng.choice(acts), bias=rng.random() < 0.75)
        if kind == "linear":
            c.update(residual=rng.random() < 0.5, keep=rng.random() < 0.5)
        else:
            c.update(act_in=rng.choice(acts))
        if work(c)["flops"] <= (1.2e12 if dtype == "bf16" else 3e10):
            return c


# ------------------------------------------------------------------------ inputs
def _shapes(c):
    """The tensors of a case's blocks: (shape, whether it decays)."""
    d, f = c["d"], c["d_ff"]
    return [((f, d), True), ((f,), False), ((d, f), True), ((d,), False), ((d,), False),
            ((d,), False)] * c["layers"]


def _spans(c):
    """Offsets of the tensors in flat buffers, each at a multiple of BLOCK, and the total."""
    at, spans = 0, []
    for shape, decays in _shapes(c):
        n = math.prod(shape)
        spans.append((at, n, shape, decays))
        at += -(-n // BLOCK) * BLOCK
    return spans, at


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        phi = torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * phi
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s = {"case": case}
    if case["kind"] == "adamw":
        spans, total = _spans(case)
        inside = torch.zeros(total, device="cuda")
        for at, n, _, _ in spans:
            inside[at:at + n] = 1
        scale = 1e-4 * torch.exp(normal(total // BLOCK, 1)).expand(-1, BLOCK).reshape(-1) * inside
        # gradients: the matrices' as the backward pass leaves them (bf16), the vectors' in fp32
        g = normal(total) * scale
        s["G"] = [g[at:at + n].view(sh).to(torch.bfloat16 if len(sh) == 2 else torch.float32)
                  for at, n, sh, _ in spans]
        m = 0.2 * normal(total) * scale
        v = (0.1 * scale * torch.exp(0.3 * normal(total))).square()
        del g, scale
        s["W"] = 0.02 * normal(total) * inside
        s["W_out"] = torch.zeros(total, device="cuda", dtype=torch.bfloat16)
        s["seed"] = 1000003 * seed + 17
        if case["bits"] == 32:
            s["m"], s["v"] = m, v
        else:
            half = torch.full((total,), 0x8000, device="cuda", dtype=torch.int64)
            s["m"], s["m_scale"] = _to_8bit(m, half, True)
            s["v"], s["v_scale"] = _to_8bit(v, half, False)
            s["m_values"], s["v_values"] = torch.empty_like(s["W_out"]), torch.empty_like(s["W_out"])
        return s
    dt, T, a, b = DTYPES[case["dtype"]], case["T"], case["d_in"], case["d_out"]
    s["W"] = (0.02 * normal(b, a)).to(dt)
    if case["kind"] == "linear":
        s["x"] = normal(T, a).to(dt)
        s["bias"] = (0.1 * normal(b)).to(dt) if case["bias"] else None
        s["residual"] = normal(T, b).to(dt) if case["residual"] else None
        s["y"] = torch.empty(T, b, device="cuda", dtype=dt)
        s["z"] = torch.empty_like(s["y"]) if case["keep"] else None
        return s
    s["dy"] = (1e-4 * normal(T, b)).to(dt)
    s["z"] = normal(T, b).to(dt) if case["act"] != "none" else None
    s["z_in"] = normal(T, a).to(dt) if case["act_in"] != "none" else None
    s["x"] = (_act(case["act_in"], s["z_in"].float()) if s["z_in"] is not None
              else normal(T, a)).to(dt)
    s["dx"] = torch.empty(T, a, device="cuda", dtype=dt)
    s["dW"] = torch.empty(b, a, device="cuda", dtype=dt)
    s["dbias"] = torch.empty(b, device="cuda") if case["bias"] else None
    return s


# ------------------------------------------------------------------------ plain forms
def _linear(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    z = s["x"].float() @ s["W"].float().t()
    z = z + s["bias"].float() if s["bias"] is not None else z
    y = _act(c["act"], z)
    y = y + s["residual"].float() if s["residual"] is not None else y
    return {"y": y.to(dt), "z": z.to(dt) if c["keep"] else None}


def _vjp(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    dz = s["dy"].float()
    dz = dz * _slope(c["act"], s["z"].float()) if s["z"] is not None else dz
    dx = dz @ s["W"].float()
    dx = dx * _slope(c["act_in"], s["z_in"].float()) if s["z_in"] is not None else dx
    return {"dx": dx.to(dt), "dW": (dz.t() @ s["x"].float()).to(dt),
            "dbias": dz.sum(0) if c["bias"] else None}


def _mix(h):
    """A bijection of 32-bit words (held in int64)."""
    h = ((h ^ (h >> 16)) * SQRT2) & WORD
    h = ((h ^ (h >> 13)) * SQRT3) & WORD
    return h ^ (h >> 16)


def _noise(seed, tensor, blocks, device):
    """32 random bits for each element of a tensor's blocks at this step."""
    key = _mix((seed + PHI) & WORD)
    key = _mix(_mix(key ^ ((seed >> 32) & WORD)) ^ STEP)
    key = _mix((key + tensor) & WORD)
    key = _mix(key ^ torch.arange(blocks, device=device))
    h = (key[:, None] + torch.arange(BLOCK, device=device) * PHI) & WORD
    h = ((h ^ (h >> 15)) * SQRT2) & WORD
    return (h ^ (h >> 16)).reshape(-1)


def _to_8bit(x, u, signed):
    """Codes and block scales of x (whole blocks), rounded up where the 16 bits u say so.
    Signed: sign, 4 exponent and 3 mantissa bits; else 5 and 3, and nothing above 0 becomes 0."""
    bias, top = (7, 7) if signed else (16, 14)
    amax = x.reshape(-1, BLOCK).abs().amax(1).clamp(min=2.0 ** -100)
    scale = torch.exp2((torch.frexp(amax)[1] - 1 - top).double()).float()
    y = x.abs().double() / scale.double().repeat_interleave(BLOCK)
    e = (torch.frexp(y)[1] - 1).clamp(min=1 - bias)
    k = torch.floor(y * torch.exp2(3.0 - e.double()) + u / 65536).long()  # 8 and more: normal numbers
    code = k + 8 * (e + bias - 1)
    if not signed:
        return torch.where(x > 0, code.clamp(min=1), code).to(torch.uint8), scale
    code = torch.where(x < 0, code + 128, code)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _from_8bit(code, scale, signed):
    scale = scale.repeat_interleave(BLOCK)
    if signed:
        return code.float() * scale
    c = code.int()
    e = (c >> 3).clamp(min=1)
    k = (c & 7) + 8 * (c >= 8).int()
    return k.float() * torch.exp2((e - 19).double()).float() * scale


def _adamw_tensor(s, k, at, n, shape, decays):
    """One tensor's step on its span of the flat buffers."""
    c, end = s["case"], -(-n // BLOCK) * BLOCK
    w = s["W"][at:at + n]
    g = s["G"][k].reshape(-1).float()
    cut, ends = slice(at, at + n), slice(at, at + end)
    if c["bits"] == 32:
        m, v = s["m"][cut], s["v"][cut]
    else:
        blocks = slice(at // BLOCK, (at + end) // BLOCK)
        m = _from_8bit(s["m"][ends], s["m_scale"][blocks], True)[:n]
        v = _from_8bit(s["v"][ends], s["v_scale"][blocks], False)[:n]
    if c["clip"] == "gradient":
        lim, norm = CLIP_FRAC * w.double().norm(), g.double().norm()
        g = g * torch.where(norm > lim, lim / norm, 1.0).float()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    wd = WEIGHT_DECAY if decays else 0.0
    mhat, den = m / (1 - BETA1 ** STEP), v.sqrt() / math.sqrt(1 - BETA2 ** STEP) + ADAM_EPS
    d = -LR * (mhat / den + wd * w)
    if c["clip"] == "step":
        lim, norm = CLIP_FRAC * w.double().norm(), d.double().norm()
        d = d * torch.where(norm > lim, lim / norm, 1.0).float()
    w.add_(d)
    s["W_out"][cut] = w.bfloat16()
    if c["bits"] == 32:
        s["m"][cut], s["v"][cut] = m, v
        return
    u = _noise(s["seed"], k, end // BLOCK, w.device)
    m, v = (torch.nn.functional.pad(x, (0, end - n)) for x in (m, v))
    mq, s["m_scale"][blocks] = _to_8bit(m, u >> 16, True)
    s["v"][ends], s["v_scale"][blocks] = _to_8bit(v, u & 0xffff, False)
    s["m"].view(torch.uint8)[ends] = mq.view(torch.uint8)


def _adamw(s):
    spans, _ = _spans(s["case"])
    _ = [_adamw_tensor(s, k, *span) for k, span in enumerate(spans)]
    out = {"W": s["W"], "W_out": s["W_out"]}
    if s["case"]["bits"] == 32:
        return {**out, "m": s["m"], "v": s["v"]}
    return {**out, "m": _from_8bit(s["m"], s["m_scale"], True).bfloat16(),
            "v": _from_8bit(s["v"], s["v_scale"], False).bfloat16()}


# ------------------------------------------------------------------------ the library's operators
def _library(s):
    import paper_2608_14563_gb300 as fpo
    c = s["case"]
    acts = {"none": fpo.ACT_NONE, "relu": fpo.ACT_RELU, "gelu": fpo.ACT_GELU,
            "gelu_tanh": fpo.ACT_GELU_TANH, "silu": fpo.ACT_SILU}
    if c["kind"] == "linear":
        fpo.linear(s["x"], s["W"], s["y"], bias=s["bias"], act=acts[c["act"]],
                   residual=s["residual"], z_out=s["z"])
        return {"y": s["y"], "z": s["z"]}
    if c["kind"] == "vjp":
        fpo.linear_vjp(s["dy"], s["x"], s["W"], s["dx"], act=acts[c["act"]], z=s["z"],
                       act_in=acts[c["act_in"]], z_in=s["z_in"], dW=s["dW"], dbias=s["dbias"])
        return {"dx": s["dx"], "dW": s["dW"], "dbias": s["dbias"]}
    clip = {"none": fpo.CLIP_NONE, "step": fpo.CLIP_STEP, "gradient": fpo.CLIP_GRADIENT}[c["clip"]]
    opt = fpo.optimizer_desc(fpo.OPT_ADAMW, lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS,
                             weight_decay=WEIGHT_DECAY, clip=clip, clip_frac=CLIP_FRAC, step=STEP)
    spans, _ = _spans(c)

    def cut(t):
        return [t[at:at + n] for at, n, _, _ in spans]

    def scales(t):
        return [t[at // BLOCK:-(-(at + n) // BLOCK)] for at, n, _, _ in spans]

    small = {}
    if c["bits"] == 8:
        small = dict(scales1=scales(s["m_scale"]), scales2=scales(s["v_scale"]), seed=s["seed"])
    fpo.adamw_grouped(s["G"], opt, cut(s["W"]), cut(s["m"]), cut(s["v"]), W_outs=cut(s["W_out"]),
                      weight_decays=[WEIGHT_DECAY if d else 0.0 for _, _, _, d in spans], **small)
    out = {"W": s["W"], "W_out": s["W_out"]}
    if c["bits"] == 32:
        return {**out, "m": s["m"], "v": s["v"]}
    # the states as numbers, as a checkpoint takes them (the tensors' spans are whole blocks)
    fpo.adamw_state_values(s["m"], s["m_scale"], s["m_values"])
    fpo.adamw_state_values(s["v"], s["v_scale"], s["v_values"])
    return {**out, "m": s["m_values"], "v": s["v_values"]}


def run(state):
    if own:
        return _library(state)
    return {"linear": _linear, "vjp": _vjp, "adamw": _adamw}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------ work and definition
def work(case):
    if case["kind"] == "adamw":
        big = sum(math.prod(sh) for sh, _ in _shapes(case) if len(sh) == 2)
        small = sum(math.prod(sh) for sh, _ in _shapes(case) if len(sh) == 1)
        n = big + small
        # masters, bf16 copy, gradients; states, for 8 bits with their values written
        state = 16 * n if case["bits"] == 32 else 8 * n + 16 * n / BLOCK
        return {"bytes": 10 * n + 2 * big + 4 * small + state, "flops": 16 * n}
    e = 2 if case["dtype"] == "bf16" else 4
    T, a, b = case["T"], case["d_in"], case["d_out"]
    bias = b if case["bias"] else 0
    if case["kind"] == "linear":
        outs = 1 + case["residual"] + case["keep"]
        return {"bytes": e * (T * a + a * b + bias + outs * T * b), "flops": 2 * T * a * b}
    ins = T * b * (1 + (case["act"] != "none")) + T * a * (1 + (case["act_in"] != "none")) + a * b
    return {"bytes": e * (ins + T * a + a * b) + 4 * bias, "flops": 4 * T * a * b}


def _exact_act(name, z):
    """act and its derivative by autograd of the definition, in fp64."""
    z = z.double().requires_grad_()
    if name == "relu":
        y = torch.where(z > 0, z, torch.zeros_like(z))
    elif name == "gelu":
        y = z * torch.special.ndtr(z)
    elif name == "gelu_tanh":
        y = z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    elif name == "silu":
        y = z / (1 + torch.exp(-z))
    else:
        y = z * 1
    (slope,) = torch.autograd.grad(y, z, torch.ones_like(y))
    return y.detach(), slope


def _exact_8bit(x, noise, bias, top, tiny):
    """The value that x (whole blocks) is kept as: the multiples of its binade's eighth beside it,
    the upper one where fraction + noise reaches 1."""
    scale = torch.exp2(torch.floor(torch.log2(x.view(-1, BLOCK).abs().amax(1).clamp(min=2.0 ** -100))) - top)
    y = (x.view(-1, BLOCK) / scale[:, None]).view(-1)
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** (1 - bias)))).clamp(min=1 - bias)
    unit = torch.exp2(e - 3)
    low = torch.floor(y.abs() / unit)
    q = (low + ((y.abs() / unit - low) + noise >= 1)) * unit
    if tiny:  # nothing above 0 is kept as 0
        q = torch.where((y > 0) & (q == 0), unit, q)
    return (torch.sign(y) * q).view(-1, BLOCK).mul(scale[:, None]).view(-1)


def _exact_bits(seed, tensor, count):
    """The noise words of a tensor's elements, by Python's integers for the keys."""
    def mix(h):
        h = (h ^ h >> 16) * SQRT2 & WORD
        h = (h ^ h >> 13) * SQRT3 & WORD
        return h ^ h >> 16
    i = torch.arange(count, device="cuda")
    key = mix(mix(mix(mix((seed + PHI) & WORD) ^ (seed >> 32 & WORD)) ^ STEP) + tensor & WORD)
    h = (mix(key ^ torch.div(i, BLOCK, rounding_mode="floor")) + (i % BLOCK) * PHI) & WORD
    h = (h ^ h >> 15) * SQRT2 & WORD
    return h ^ h >> 16


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        z = torch.nn.functional.linear(s["x"].double(), s["W"].double(),
                                       s["bias"].double() if case["bias"] else None)
        y, _ = _exact_act(case["act"], z)
        y = y + s["residual"].double() if case["residual"] else y
        return {"y": y, "z": z if case["keep"] else None}
    if case["kind"] == "vjp":
        dz = s["dy"].double()
        if s["z"] is not None:
            dz = dz * _exact_act(case["act"], s["z"])[1]
        dx = torch.einsum("to,oi->ti", dz, s["W"].double())
        if s["z_in"] is not None:
            dx = dx * _exact_act(case["act_in"], s["z_in"])[1]
        return {"dx": dx, "dW": torch.einsum("to,ti->oi", dz, s["x"].double()),
                "dbias": torch.einsum("to->o", dz) if case["bias"] else None}
    spans, _ = _spans(case)
    W, M = s["W"].double(), torch.zeros_like(s["W"], dtype=torch.float64)
    V = torch.zeros_like(M)
    for k, (at, n, _, decays) in enumerate(spans):
        cut, ends = slice(at, at + n), slice(at, at + -(-n // BLOCK) * BLOCK)
        w, g = W[cut], s["G"][k].double().view(-1)
        if case["bits"] == 32:
            m, v = s["m"][cut].double(), s["v"][cut].double()
        else:
            sc = slice(ends.start // BLOCK, ends.stop // BLOCK)
            m = (s["m"][ends].double().view(-1, BLOCK) * s["m_scale"][sc].double()[:, None]).view(-1)[:n]
            code = s["v"][ends].double()
            e = torch.floor(code / 8)
            val = torch.where(e > 0, (code - 8 * e + 8) * torch.exp2(e - 19), code * 2.0 ** -18)
            v = (val.view(-1, BLOCK) * s["v_scale"][sc].double()[:, None]).view(-1)[:n]
        ratio = CLIP_FRAC * torch.linalg.vector_norm(w)
        if case["clip"] == "gradient":
            g = g * torch.clamp(ratio / torch.linalg.vector_norm(g), max=1.0)
        m = torch.lerp(g, m, BETA1)
        v = torch.lerp(g * g, v, BETA2)
        d = (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + ADAM_EPS)
        d = LR * (d + (WEIGHT_DECAY if decays else 0.0) * w)
        if case["clip"] == "step":
            d = d * torch.clamp(ratio / torch.linalg.vector_norm(d), max=1.0)
        W[cut] = w - d
        if case["bits"] == 32:
            M[cut], V[cut] = m, v
            continue
        u, pad = _exact_bits(s["seed"], k, ends.stop - at), (0, ends.stop - at - n)
        m, v = torch.nn.functional.pad(m, pad), torch.nn.functional.pad(v, pad)
        M[ends] = _exact_8bit(m, (u >> 16) / 65536, 7, 7, False)
        V[ends] = _exact_8bit(v, (u & 0xffff) / 65536, 16, 14, True)
    return {"W": W, "W_out": W, "m": M, "v": V}
