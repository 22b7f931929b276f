"""Measured cases of the LayerNorm and Newton-Schulz (Muon) operators.

Kinds:

* ``ln_fwd``   LayerNorm forward: y, and per token the mean and 1 / sigma
* ``ln_vjp``   its backward pass: the signal through the norm's Jacobian, and the gradients
               of the weight and the bias
* ``orth``     orthogonalised updates: five Newton-Schulz steps on every layer's matrix
* ``muon``     the optimizer step of target layers: pseudogradient, momentum, Newton-Schulz,
               weight update

``run`` computes them in elementary torch operations in fp32, or, with ``own`` set, through
the library's entry points.  ``exact`` states the same definitions once more in fp64.

Sizes are those of the repository's workloads and tests, or generic ones of the same ranges.
Inputs follow the distributions of the workloads: x ~ per-token scaled normal, weights
gamma = 1 + 0.1 N, A = SiLU(N) N, W ~ N(0, 0.02^2), signals of the size that a mean-reduced
cross-entropy leaves.
"""
import math

import torch

own = False

LN_EPS, MIN_RMS = 1e-5, 0.5
NS_STEPS, NS_EPS = 5, 1e-7
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315
MU, WEIGHT_DECAY = 0.95, 0.1
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------ the cases
def listed():
    return [
        # one token's hidden state, as a token-by-token forward pass normalises it: launch latency
        dict(name="ln-fwd-one-token", kind="ln_fwd", dtype="bf16", T=1, d=4096),
        # the training batch of the 7B-shaped workload: 8 packed 2048-token sequences
        dict(name="ln-fwd-training-batch", kind="ln_fwd", dtype="bf16", T=16384, d=4096),
        # a short ragged document at a small model's width
        dict(name="ln-vjp-short", kind="ln_vjp", dtype="bf16", T=200, d=256),
        # the training batch's backward pass
        dict(name="ln-vjp-training-batch", kind="ln_vjp", dtype="bf16", T=16384, d=4096),
        # an fp32 reference run with odd sizes: rows that are not aligned to 16 bytes
        dict(name="ln-vjp-f32-odd", kind="ln_vjp", dtype="f32", T=4097, d=1023),
        # the two matrices of a unit-test-sized model: a chain of launches
        dict(name="orth-small", kind="orth", dtype="bf16", rows=256, cols=384, layers=2, T=200),
        # one down-projection of the 7B shape, its gradient from one packed sequence
        # (half of the row space only)
        dict(name="orth-7b-layer", kind="orth", dtype="bf16", rows=4096, cols=11008, layers=1,
             T=2048),
        # an fp32 reference run at a small model's size, odd sizes
        dict(name="orth-f32-odd", kind="orth", dtype="f32", rows=767, cols=2049, layers=2, T=4096),
        # the fp32 workload of the test-suite
        dict(name="muon-f32-tiny", kind="muon", dtype="f32", T=128, d=64, d_ff=256, layers=2),
        # a short bf16 step with a ragged token count
        dict(name="muon-short", kind="muon", dtype="bf16", T=200, d=256, d_ff=384, layers=2),
        # gate and up matrices (taller than wide) of a 1B-sized model on one packed sequence
        dict(name="muon-gate-up", kind="muon", dtype="bf16", T=2048, d=8192, d_ff=2048, layers=2),
        # two target layers of the 7B shape on two packed sequences
        dict(name="muon-7b-layers", kind="muon", dtype="bf16", T=4096, d=4096, d_ff=11008,
             layers=2),
    ]


def _log(rng, lo, hi, mult=1):
    """A size spread over the logarithm of [lo, hi], a multiple of mult."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / mult)) * mult, -(-lo // mult) * mult), hi // mult * mult)


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_vjp", "ln_vjp", "orth", "orth", "muon", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    mult = 8 if dtype == "bf16" else 1
    if kind in ("ln_fwd", "ln_vjp"):
        while True:
            c = dict(kind=kind, dtype=dtype, T=_log(rng, 1, 32768), d=_log(rng, 32, 12288, mult))
            if c["T"] * c["d"] * (2 if dtype == "bf16" else 4) <= 16384 * 4096 * 2:
                return c
    # fp32 matrices up to a small model's size; their gradients have full rank
    lo, hi = (16, 8192) if dtype == "bf16" else (16, 1536)
    while True:
        rows, cols = _log(rng, lo, hi, mult), _log(rng, lo, hi, mult)
        m, layers = min(rows, cols), rng.choice([1, 1, 2, 3, 4])
        T = _log(rng, 1, 8192) if dtype == "bf16" else _log(rng, 4 * m, 8 * m)
        if kind == "orth":
            c = dict(kind=kind, dtype=dtype, rows=rows, cols=cols, layers=layers, T=T)
        else:
            c = dict(kind=kind, dtype=dtype, T=T, d=rows, d_ff=cols, layers=layers)
        if work(c)["flops"] <= 0.5 * work(listed()[-1])["flops"]:
            return c


# ------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    gen, dt = _gen(seed), DTYPES[case["dtype"]]
    f32 = dict(device="cuda", dtype=torch.float32)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s = {"case": case}
    if case["kind"] in ("ln_fwd", "ln_vjp"):
        T, d = case["T"], case["d"]
        # per-token scale spread over a factor of several, a mean off zero
        scale = torch.exp(0.5 * normal(T, 1))
        s["x"] = (normal(T, d) * scale + 0.2 * scale).to(dt)
        s["gamma"] = (1 + 0.1 * normal(d)).to(dt)
        s["beta"] = (0.1 * normal(d)).to(dt)
        s["out"] = torch.empty(T, d, device="cuda", dtype=dt)
        if case["kind"] == "ln_fwd":
            s["mean"], s["rstd"] = torch.empty(T, **f32), torch.empty(T, **f32)
        else:
            s["g"] = (1e-2 * normal(T, d)).to(dt)
            s["dgamma"], s["dbeta"] = torch.empty(d, **f32), torch.empty(d, **f32)
        return s
    T, n = case["T"], case["layers"]
    rows, cols = (case["rows"], case["cols"]) if case["kind"] == "orth" else (case["d"], case["d_ff"])
    gs = [(1e-4 * normal(T, rows)).to(dt) for _ in range(n)]
    As = [(torch.nn.functional.silu(normal(T, cols)) * normal(T, cols)).to(dt) for _ in range(n)]
    if case["kind"] == "orth":
        s["G"] = [(g.float().t() @ a.float()).to(dt) for g, a in zip(gs, As)]
        s["O"] = [torch.empty_like(G) for G in s["G"]]
        return s
    s["g"], s["A"] = gs, As
    s["M"] = [6e-5 * math.sqrt(T) * normal(rows, cols) for _ in range(n)]
    s["W"] = [0.02 * normal(rows, cols) for _ in range(n)]
    s["W_out"] = [torch.empty(rows, cols, device="cuda", dtype=dt) for _ in range(n)]
    # the step's root mean square matches an AdamW step of this rate times 0.2
    s["lr"], s["scale"] = 5e-5, 0.2 * math.sqrt(max(rows, cols))
    return s


# ------------------------------------------------------------------------ plain forms
def _newton_schulz(G):
    X = G.float()
    X = X / X.square().sum().sqrt().clamp(min=NS_EPS)
    tall = X.shape[0] > X.shape[1]
    X = X.t() if tall else X
    for _ in range(NS_STEPS):
        A = X @ X.t()
        X = NS_A * X + (NS_B * A + NS_C * (A @ A)) @ X
    return X.t() if tall else X


def _ln_fwd(s):
    x, w, b = s["x"].float(), s["gamma"].float(), s["beta"].float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1 / (xc.square().mean(1, keepdim=True) + LN_EPS).sqrt()
    y = (xc * rstd * w + b).to(s["x"].dtype)
    return {"y": y, "mean": mean.squeeze(1), "rstd": rstd.squeeze(1)}


def _ln_vjp(s):
    g, x, w = s["g"].float(), s["x"].float(), s["gamma"].float()
    xc = x - x.mean(1, keepdim=True)
    sigma = (xc.square().mean(1, keepdim=True) + LN_EPS).sqrt()
    xh = xc / sigma
    u = g * w
    out = u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True)
    out = out / sigma.clamp(min=MIN_RMS)
    return {"g_out": out.to(s["x"].dtype), "dgamma": (g * xh).sum(0), "dbeta": g.sum(0)}


def _muon_layer(g, A, M, W, dt, lr, scale):
    G = g.float().t() @ A.float()
    M.mul_(MU).add_(G)
    O = _newton_schulz(G + MU * M)
    W.mul_(1 - lr * WEIGHT_DECAY).sub_(lr * scale * O)
    return W.to(dt)


def _plain(s):
    kind, dt = s["case"]["kind"], DTYPES[s["case"]["dtype"]]
    if kind == "ln_fwd":
        return _ln_fwd(s)
    if kind == "ln_vjp":
        return _ln_vjp(s)
    if kind == "orth":
        return {"O": [_newton_schulz(G).to(dt) for G in s["G"]]}
    W_out = [_muon_layer(g, A, M, W, dt, s["lr"], s["scale"])
             for g, A, M, W in zip(s["g"], s["A"], s["M"], s["W"])]
    return {"M": s["M"], "W": s["W"], "W_out": W_out}


# ------------------------------------------------------------------------ the library's operators
def _library(s):
    import paper_2608_14563_gb300 as fpo
    kind = s["case"]["kind"]
    if kind == "ln_fwd":
        fpo.layernorm(s["x"], s["gamma"], s["beta"], s["out"], eps=LN_EPS, mean_out=s["mean"],
                      rstd_out=s["rstd"])
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    if kind == "ln_vjp":
        fpo.layernorm_vjp(s["g"], s["x"], s["gamma"], s["out"], eps=LN_EPS, min_rms=MIN_RMS,
                          dgamma=s["dgamma"], dbeta=s["dbeta"])
        return {"g_out": s["out"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if kind == "orth":
        fpo.orthogonalize_grouped(s["G"], s["O"], steps=NS_STEPS, eps=NS_EPS)
        return {"O": s["O"]}
    opt = fpo.muon_desc(lr=s["lr"], momentum=MU, weight_decay=WEIGHT_DECAY, scale=s["scale"],
                        nesterov=True, steps=NS_STEPS, eps=NS_EPS)
    fpo.layer_muon_grouped(s["g"], s["A"], opt, s["W"], s["M"], W_outs=s["W_out"])
    return {"M": s["M"], "W": s["W"], "W_out": s["W_out"]}


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------------ work and definition
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    n = case.get("layers", 1)
    if case["kind"] == "ln_fwd":
        T, d = case["T"], case["d"]
        return {"bytes": 2 * T * d * e + 2 * d * e + 8 * T, "flops": 8 * T * d}
    if case["kind"] == "ln_vjp":
        T, d = case["T"], case["d"]
        return {"bytes": 3 * T * d * e + d * e + 8 * d, "flops": 16 * T * d}
    rows, cols = (case["rows"], case["cols"]) if case["kind"] == "orth" else (case["d"], case["d_ff"])
    m, k = min(rows, cols), max(rows, cols)
    # A and A^2 are symmetric: half of each product
    ns = NS_STEPS * (m * m * k + m ** 3 + 2 * m * m * k)
    if case["kind"] == "orth":
        return {"bytes": n * 2 * m * k * e, "flops": n * ns}
    T = case["T"]
    return {"bytes": n * (T * (m + k) * e + m * k * (16 + e)), "flops": n * (2 * T * m * k + ns)}


def _exact_orth(U):
    """p(sigma) of every singular value, p five times a s + b s^3 + c s^5, from the products of
    the matrix with its transpose in fp64."""
    Y = U / max(float(torch.linalg.vector_norm(U)), NS_EPS)
    wide = Y.shape[0] <= Y.shape[1]
    eye = torch.eye(min(Y.shape), device=Y.device, dtype=Y.dtype)
    for _ in range(NS_STEPS):
        S = Y @ Y.mT if wide else Y.mT @ Y
        P = torch.addmm(NS_B * S, S, S, alpha=NS_C) + NS_A * eye
        Y = P @ Y if wide else Y @ P
    return Y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("ln_fwd", "ln_vjp"):
        x, w = s["x"].double(), s["gamma"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        sigma = torch.sqrt(var + LN_EPS)
        z = (x - mean[:, None]) / sigma[:, None]
        if case["kind"] == "ln_fwd":
            return {"y": torch.addcmul(s["beta"].double(), z, w), "mean": mean, "rstd": 1 / sigma}
        g, d = s["g"].double(), case["d"]
        u = g * w
        # the Jacobian's two projections, off 1 and off z
        c0, c1 = u.sum(1) / d, torch.einsum("td,td->t", u, z) / d
        out = (u - c0[:, None] - c1[:, None] * z) / torch.clamp(sigma, min=MIN_RMS)[:, None]
        return {"g_out": out, "dgamma": torch.einsum("td,td->d", g, z), "dbeta": g.sum(0)}
    if case["kind"] == "orth":
        return {"O": [_exact_orth(G.double()) for G in s["G"]]}
    M, W = [], []
    for g, A, m0, w0 in zip(s["g"], s["A"], s["M"], s["W"]):
        G = torch.einsum("ti,tj->ij", g.double(), A.double())
        M.append(torch.add(G, m0.double(), alpha=MU))
        O = _exact_orth(torch.add(G, M[-1], alpha=MU))
        W.append(w0.double() * (1 - s["lr"] * WEIGHT_DECAY) - s["lr"] * s["scale"] * O)
    return {"M": M, "W": W, "W_out": W}
