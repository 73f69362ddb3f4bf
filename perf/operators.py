"""Operators measured on their own: orthogonalising an update by Newton-Schulz
products, the optimizer step built on it, and layer norm forward and backward
with the gradients of its gain and bias, over the range of sizes a user of the
framework runs them at.

listed() names the fixed cases, draw(rng) gives one more of the same ranges,
prepare / run / exact make the inputs, one pass and its float64 result, work
states what a pass cannot do without. With `own` false, run computes the
operators in elementary torch operations; with it true, by the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NS_EPS, NS_COEF = 1e-7, (3.4445, -4.7750, 2.0315)
LN_EPS = 1e-5
LR, MOMENTUM, WEIGHT_DECAY = 1e-4, 0.9, 0.01


# --------------------------------------------------------------------- the cases
def listed() -> list:
    return [
        # the down projections of the smallest configuration, at the parity precision: launches and latency
        dict(name="orth f32 tiny", kind="orth", dtype="f32", rows=256, cols=688, n=2, steps=5),
        # four matrices of which no side is a whole tile
        dict(name="orth bf16 ragged", kind="orth", dtype="bf16", rows=1000, cols=2744, n=4, steps=5),
        # gate and up projection of one OLMo-2-7B layer (more rows than columns)
        dict(name="orth bf16 tall olmo2", kind="orth", dtype="bf16", rows=11008, cols=4096, n=2, steps=5),
        # the step on the small end-to-end diagnostic model's down projections
        dict(name="muon f32 small", kind="muon", dtype="f32", rows=384, cols=1032, n=3, steps=5),
        # a model of about a billion parameters: its last six layers
        dict(name="muon bf16 1b", kind="muon", dtype="bf16", rows=2048, cols=5504, n=6, steps=5),
        # the optimizer step of a Qwen3-8B training step: its nine target layers
        dict(name="muon bf16 qwen3", kind="muon", dtype="bf16", rows=4096, cols=12288, n=9, steps=5),
        # one token (decoding)
        dict(name="ln bf16 one token", kind="ln", dtype="bf16", T=1, d=4096),
        # the parity precision at a ragged size, with the rows' statistics
        dict(name="ln f32 ragged", kind="ln", dtype="f32", T=611, d=1032, stats=True),
        # the layer-viability diagnostic's 16 x 512 tokens
        dict(name="ln bf16 8192 tokens", kind="ln", dtype="bf16", T=8192, d=4096),
        # a short sequence: few rows, the gradients of gain and bias dominate
        dict(name="ln vjp bf16 short", kind="ln_vjp", dtype="bf16", dy="bf16", T=48, d=2048, min_std=0.0),
        # float32 everywhere, nothing a power of two
        dict(name="ln vjp f32 ragged", kind="ln_vjp", dtype="f32", dy="f32", T=1999, d=2568, min_std=0.0),
        # the final norm of a training step: float32 error signal, clamped, float32 and bf16 results
        dict(name="ln vjp bf16 8192 tokens", kind="ln_vjp", dtype="bf16", dy="f32", T=8192, d=4096, min_std=0.5),
    ]


def _log_int(rng, lo: int, hi: int, step: int = 1) -> int:
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng) -> dict:
    kind = rng.choice(["orth", "muon", "ln", "ln_vjp"])
    f32 = rng.random() < 0.3
    dtype = "f32" if f32 else "bf16"
    if kind in ("orth", "muon"):
        a = _log_int(rng, 64, 1536 if f32 else 4096, 8)
        b = min(12288, int(a * rng.uniform(1.0, 4.0)) // 8 * 8)
        rows, cols = (a, b) if rng.random() < 0.6 else (b, a)
        c = dict(kind=kind, dtype=dtype, rows=rows, cols=cols, n=rng.randint(1, 9), steps=rng.choice([5, 5, 5, 4, 6]))
        while c["n"] > 1 and work(c)["flops"] > (1e12 if f32 else 1.2e13):
            c["n"] -= 1
        return c
    c = dict(kind=kind, dtype=dtype, T=_log_int(rng, 1, 16384), d=_log_int(rng, 64, 8192, 8))
    if kind == "ln":
        c["stats"] = rng.random() < 0.5
    else:
        c["dy"] = "f32" if f32 or rng.random() < 0.5 else "bf16"
        c["min_std"] = rng.choice([0.0, 0.5])
    return c


# --------------------------------------------------------------------- inputs
class _Draw:
    def __init__(self, seed: int):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(mean, std, generator=self.g)

    def gradient(self, rows, cols, tokens):
        """A token-summed outer product of an error signal (tokens of unequal
        weight) with a SwiGLU activation, as the pseudogradients are."""
        n, m = min(rows, cols), max(rows, cols)
        g = self.normal((tokens, n), 0.02).mul_(self.normal((tokens, 1), 0.5).exp_())
        a = torch.nn.functional.silu(self.normal((tokens, m))).mul_(self.normal((tokens, m)))
        D = (g.t().contiguous().bfloat16() @ a.bfloat16()).float().div_(tokens)
        return D if rows <= cols else D.t().contiguous()

    def hidden(self, T, d):
        """Hidden states: an offset and a scale for each token, 1% of the
        channels twenty times larger, 1% of the tokens (the first among them)
        nearly constant."""
        s = self.normal((T, 1), 0.3).exp_()
        s[::100] = 0.05
        x = self.normal((T, d)).mul_(s).add_(self.normal((T, 1), 0.3))
        x[:, ::97] *= 20.0
        return x


def prepare(case: dict, seed: int) -> dict:
    c, r = case, _Draw(seed)
    s = dict(case=c)
    op = DT[c["dtype"]]
    if c["kind"] in ("orth", "muon"):
        R, C, n = c["rows"], c["cols"], c["n"]
        small = min(R, C)
        if c["kind"] == "orth":
            s["X"] = [r.gradient(R, C, 2 * small).to(op) for _ in range(n)]
            s["O"] = [torch.empty(R, C, dtype=op, device=DEV) for _ in range(n)]
        else:
            s["grad"] = [r.gradient(R, C, small) for _ in range(n)]
            s["state"] = [r.gradient(R, C, 2 * small).mul_(5.0) for _ in range(n)]
            s["W"] = [r.normal((R, C), 0.02) for _ in range(n)]
            s["W_lp"] = [torch.empty(R, C, dtype=op, device=DEV) for _ in range(n)]
        return s
    T, d = c["T"], c["d"]
    s.update(x=r.hidden(T, d).to(op), gain=r.normal((d,), 0.1, 1.0).to(op))
    if c["kind"] == "ln":
        s.update(bias=r.normal((d,), 0.1).to(op), y=torch.empty(T, d, dtype=op, device=DEV), mean=None, rstd=None)
        if c.get("stats"):
            s.update(mean=torch.empty(T, device=DEV), rstd=torch.empty(T, device=DEV))
    else:
        s.update(dy=r.normal((T, d), 0.02).to(DT[c["dy"]]), dx=torch.empty(T, d, device=DEV), dx_lp=None,
                 dgain=torch.empty(d, device=DEV), dbias=torch.empty(d, device=DEV))
        if c["dtype"] == "bf16":
            s["dx_lp"] = torch.empty(T, d, dtype=op, device=DEV)
    return s


# --------------------------------------------------------------------- the plain forms
def _newton_schulz(X, steps):
    """X in float32, rows <= columns. Its norm is a long sum: in 64 bits."""
    a, b, c = NS_COEF
    X = (X.double() / (X.double().square().sum().sqrt() + NS_EPS)).float()
    for _ in range(steps):
        A = X @ X.t()
        B = b * A + c * (A @ A)
        X = a * X + B @ X
    return X


def _orthogonal(M, steps):
    M = M.float()
    return _newton_schulz(M, steps) if M.shape[0] <= M.shape[1] else _newton_schulz(M.t(), steps).t()


def _scale(rows, cols):
    return 0.2 * math.sqrt(max(rows, cols))


def _plain_muon(s, m):
    """One matrix's step; state, master and its low-precision copy in place."""
    c = s["case"]
    g, buf, W = s["grad"][m], s["state"][m], s["W"][m]
    buf.mul_(MOMENTUM).add_(g)
    O = _orthogonal(g + MOMENTUM * buf, c["steps"])
    W.mul_(1.0 - LR * WEIGHT_DECAY).sub_(O.mul(LR * _scale(c["rows"], c["cols"])))
    s["W_lp"][m].copy_(W)


def _plain_ln(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / ((x - mean).square().mean(1, keepdim=True) + LN_EPS).sqrt()
    y = (x - mean) * rstd * s["gain"].float() + s["bias"].float()
    return y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]


def _plain_ln_vjp(s):
    x, dy = s["x"].float(), s["dy"].float()
    xc = x - x.mean(1, keepdim=True)
    std = (xc.square().mean(1, keepdim=True) + LN_EPS).sqrt()
    dgain = (dy * (xc / std)).sum(0)
    dbias = dy.sum(0)
    std = std.clamp(min=s["case"]["min_std"])
    xh, v = xc / std, dy * s["gain"].float()
    dx = (v - v.mean(1, keepdim=True) - xh * (v * xh).mean(1, keepdim=True)) / std
    return dx, dgain, dbias


# --------------------------------------------------------------------- one pass
def run(state: dict):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "orth":
        return {"O": [_orthogonal(X, c["steps"]).to(X.dtype) for X in s["X"]]}
    if c["kind"] == "muon":
        for m in range(c["n"]):
            _plain_muon(s, m)
        return {"W": s["W"], "W_lp": s["W_lp"], "state": s["state"]}
    if c["kind"] == "ln":
        y, mean, rstd = _plain_ln(s)
        return {"y": y, "mean": mean, "rstd": rstd} if c.get("stats") else {"y": y}
    dx, dgain, dbias = _plain_ln_vjp(s)
    out = {"dx": dx, "dgain": dgain, "dbias": dbias}
    if s["dx_lp"] is not None:
        out["dx_lp"] = dx.to(s["dx_lp"].dtype)
    return out


def _run_own(s, c):
    from paper_2608_14563_amd import api

    # the workspace is made by the first pass and kept, as a training loop keeps it
    if c["kind"] == "orth":
        s["ws"] = api.fpo_orthogonalize(s["X"], s["O"], steps=c["steps"], eps=NS_EPS, ws=s.get("ws"))
        return {"O": s["O"]}
    if c["kind"] == "muon":
        opt = api.MuonConfig(lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=WEIGHT_DECAY, clip_frac=0.0, step=7,
                             scale=api.MUON_SCALE_RMS, steps=c["steps"], eps=NS_EPS)
        s["ws"] = api.fpo_muon_update(opt, s["grad"], s["W"], s["state"], W_lp=s["W_lp"], dtype=DT[c["dtype"]],
                                      ws=s.get("ws"))
        return {"W": s["W"], "W_lp": s["W_lp"], "state": s["state"]}
    if c["kind"] == "ln":
        api.fpo_layernorm(s["x"], s["gain"], s["bias"], s["y"], mean=s["mean"], rstd=s["rstd"], eps=LN_EPS)
        return {k: s[k] for k in (("y", "mean", "rstd") if c.get("stats") else ("y",))}
    s["ws"] = api.fpo_layernorm_vjp(s["x"], s["gain"], s["dy"], dx=s["dx"], dx_lp=s["dx_lp"], dgain=s["dgain"],
                                    dbias=s["dbias"], eps=LN_EPS, min_std=c["min_std"], ws=s.get("ws"))
    return {k: s[k] for k in ("dx", "dx_lp", "dgain", "dbias") if s[k] is not None}


# --------------------------------------------------------------------- what a pass cannot do without
def work(case: dict) -> dict:
    c = case
    esz = 2.0 if c["dtype"] == "bf16" else 4.0
    if c["kind"] in ("orth", "muon"):
        n, m, k = min(c["rows"], c["cols"]), max(c["rows"], c["cols"]), c["steps"]
        # the fewest operations known here: the steps' polynomials of the n x n Gram matrix (symmetric, half of each
        # product: A A, two for the next A, one for the product of the polynomials), its own product and the last one
        f = 3.0 * n * n * m + (4 * k - 3) * float(n) ** 3
        # orth: read and written once. muon: gradient read, momentum and master read and written, the copy written
        b = n * m * (2 * esz if c["kind"] == "orth" else 4.0 + 8.0 + 8.0 + esz)
        return {"bytes": b * c["n"], "flops": f * c["n"]}
    T, d = c["T"], c["d"]
    if c["kind"] == "ln":
        return {"bytes": esz * (2.0 * T * d + 2 * d) + (8.0 * T if c.get("stats") else 0.0), "flops": 8.0 * T * d}
    lp = 2.0 if c["dtype"] == "bf16" else 0.0
    return {"bytes": T * d * (esz + (4.0 if c["dy"] == "f32" else 2.0) + 4.0 + lp) + d * (esz + 8.0),
            "flops": 18.0 * T * d}


# --------------------------------------------------------------------- float64 results
def _exact_orthogonal(M, steps):
    """a X + b (X X^T) X + c (X X^T)^2 X at every step, by products with X alone."""
    M = M.double()
    X = M if M.shape[0] <= M.shape[1] else M.t().contiguous()
    X = X / (torch.linalg.matrix_norm(X) + NS_EPS)
    a, b, c = NS_COEF
    for _ in range(steps):
        G = X @ X.t()
        X1 = G @ X
        X = a * X + b * X1 + c * (G @ X1)
    return X if M.shape[0] <= M.shape[1] else X.t()


def exact(case: dict, seed: int):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "orth":
        return {"O": [_exact_orthogonal(X, c["steps"]) for X in s["X"]]}
    if c["kind"] == "muon":
        W, S = [], []
        for g, b, w in zip(s["grad"], s["state"], s["W"]):
            b = MOMENTUM * b.double() + g.double()
            O = _exact_orthogonal(g.double() + MOMENTUM * b, c["steps"])
            S.append(b.float())
            W.append((w.double() * (1 - LR * WEIGHT_DECAY) - LR * _scale(c["rows"], c["cols"]) * O).float())
        return {"W": W, "W_lp": W, "state": S}
    x, gain = s["x"].double(), s["gain"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    std = (var + LN_EPS).sqrt()
    xh = (x - mean) / std
    if c["kind"] == "ln":
        out = {"y": xh * gain + s["bias"].double()}
        if c.get("stats"):
            out.update(mean=mean[:, 0], rstd=1.0 / std[:, 0])
        return out
    dy = s["dy"].double()
    out = {"dgain": torch.linalg.vecdot(dy, xh, dim=0), "dbias": dy.sum(0)}
    k = std.clamp(min=c["min_std"])
    xk, v = xh * (std / k), dy * gain
    d = c["d"]
    out["dx"] = (v - v.sum(1, keepdim=True) / d - xk * torch.linalg.vecdot(v, xk, dim=1)[:, None] / d) / k
    if s["dx_lp"] is not None:
        out["dx_lp"] = out["dx"]
    return out
