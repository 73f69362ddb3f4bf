"""A training step of one target layer in a layer-norm model, the calls as they are used
together: layer norm forward on the residual stream, its VJP for the error signal with
the gradients of gain and bias, the signal's outer product with the layer's activation,
the Muon step on that matrix (clipped to 1% of it) and the AdamW step on gain and bias.
Three steps against float64; eager, and captured once and replayed.

Tolerances: relative Frobenius errors of what the calls' own tests allow them, summed
along the chain. FPO_BF16: signal and activations are bf16, 2^-9 a rounding on average;
orthogonalising enlarges what is off in directions whose singular value is a tenth of the
others', as the smallest of this gradient are (136 rows from 200 tokens of unequal weight),
ten times, so that the direction is off by 2% at most; the step it scales is 1% of W, three
steps 3 x 2e-2 x 1e-2. FPO_F32: products to 2^-22, sums over 200 tokens, the direction to
1e-4 for the same reason."""
import threading

import numpy as np
import pytest
import torch

from oracle import operators as P
from paper_2608_14563_amd import _lib as L
from paper_2608_14563_amd import api
from tests._util import host64, rel_fro

pytestmark = pytest.mark.gpu
T, D, F = 200, 136, 328


def make(dev, dtype, seed=0):
    rng = np.random.default_rng(seed)
    t = lambda a, dt=torch.float32: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev).to(dt)  # noqa: E731
    x = rng.normal(size=(T, D)) * np.exp(0.5 * rng.normal(size=(T, 1))) + 0.3
    x[::50] *= 0.02  # rows under the floor
    q, u = rng.normal(size=(2, T, F))
    s = dict(x=t(x, dtype), a=t(q / (1 + np.exp(-q)) * u, dtype), dy=t(0.02 * rng.normal(size=(T, D))),
             gain=t(1 + 0.1 * rng.normal(size=D)), bias=t(0.1 * rng.normal(size=D)), W=t(0.02 * rng.normal(size=(D, F))))
    z = lambda *n: torch.zeros(*n, device=dev)  # noqa: E731
    s.update(gain_lp=s["gain"].to(dtype), bias_lp=s["bias"].to(dtype), y=z(T, D).to(dtype), dx=z(T, D), dx_lp=z(T, D).to(dtype),
             dgain=z(D), dbias=z(D), dW=z(D, F), mom=z(D, F), m1=[z(D), z(D)], m2=[z(D), z(D)], W_lp=z(D, F).to(dtype),
             ss=z(1).double(), psq=z(2).double(), clip=z(1))
    s["W_sumsq"] = (s["W"].double() ** 2).sum().reshape(1)
    s["p_sumsq"] = torch.stack([(s[k].double() ** 2).sum() for k in ("gain", "bias")])
    s["ws"] = dict(vjp=api.workspace(api.fpo_layernorm_vjp_workspace(T, D), dev),
                   pg=api.workspace(api.fpo_pseudograd_workspace(T, D, F, 1, dtype), dev),
                   mu=api.workspace(api.fpo_muon_update_workspace([(D, F)], dtype), dev),
                   cos=api.workspace(api.fpo_cosine_workspace([D, D]), dev),
                   up=api.workspace(api.fpo_apply_update_workspace([D, D]), dev))
    return s


MUON = dict(lr=2e-2, momentum=0.9, weight_decay=0.01, clip_frac=0.01, clip_target=L.FPO_CLIP_UPDATE)
ADAM = dict(kind=L.FPO_OPT_ADAMW, lr=1e-3, clip_frac=0.0)


def step(s, k, dtype):
    ws = s["ws"]
    api.fpo_layernorm(s["x"], s["gain_lp"], s["bias_lp"], s["y"])
    api.fpo_layernorm_vjp(s["x"], s["gain_lp"], s["dy"], dx=s["dx"], dx_lp=s["dx_lp"], dgain=s["dgain"], dbias=s["dbias"],
                          min_std=0.5, ws=ws["vjp"])
    api.fpo_pseudograd(s["dx_lp"], [s["a"]], dW3=[s["dW"]], sumsq=s["ss"], ws=ws["pg"])
    api.fpo_muon_update(api.MuonConfig(step=k, **MUON), [s["dW"]], [s["W"]], [s["mom"]], W_sumsq=s["W_sumsq"],
                        W_lp=[s["W_lp"]], clip_scale=s["clip"], dtype=dtype, ws=ws["mu"])
    grads = [s["dgain"], s["dbias"]]
    api.fpo_cosine(grads, sumsq_A=s["psq"], ws=ws["cos"])
    api.fpo_apply_update(api.OptConfig(step=k, **ADAM), grads, s["psq"], [s["gain"], s["bias"]], s["m1"], s["p_sumsq"],
                         W_lp=[s["gain_lp"], s["bias_lp"]], state2=s["m2"], lp_dtype=dtype, ws=ws["up"])


def reference(s, steps):
    x, a, dy = host64(s["x"]), host64(s["a"]), host64(s["dy"])
    gain, bias, W = host64(s["gain"]), host64(s["bias"]), host64(s["W"])
    low = lambda v: host64(torch.from_numpy(v).to(s["x"].dtype))  # noqa: E731  (what the calls read of gain and bias)
    mom, m1, m2 = np.zeros_like(W), [0.0, 0.0], [0.0, 0.0]
    for k in range(1, steps + 1):
        g = low(gain)
        y = P.layernorm(x, g, low(bias))[0]
        dx, dg, db = P.layernorm_vjp(x, g, dy, min_std=0.5)
        dW = dx.T @ a / T
        W, mom, clip, _ = P.muon(W, dW, mom, MUON["lr"], MUON["momentum"], True, MUON["weight_decay"], "rms", k,
                                 MUON["clip_frac"], "update")
        new = []
        for i, (p, d) in enumerate(((gain, dg), (bias, db))):
            m1[i] = 0.9 * m1[i] + 0.1 * d
            m2[i] = 0.999 * m2[i] + 0.001 * d * d
            st = m1[i] / (1 - 0.9 ** k) / (np.sqrt(m2[i] / (1 - 0.999 ** k)) + 1e-8)
            new.append(p * (1 - 1e-3 * 0.01) - 1e-3 * st)
        gain, bias = new
    return dict(y=y, dx=dx, dgain=dg, dbias=db, dW=dW, W=W, mom=mom, gain=gain, bias=bias), clip


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_three_steps(dev, dtype):
    s = make(dev, dtype)
    ref, clip = reference(s, 3)
    for k in (1, 2, 3):
        step(s, k, dtype)
    assert clip < 1 and abs(float(s["clip"]) - clip) < (2e-2 if dtype == torch.bfloat16 else 1e-4) * clip
    if dtype == torch.bfloat16:
        tol = dict(y=2 ** -8, dx=1e-4, dgain=1e-4, dbias=1e-4, dW=2 ** -8, mom=2 ** -8, W=6e-4, gain=1e-4, bias=1e-4)
    else:
        tol = dict(y=1e-6, dx=1e-5, dgain=1e-5, dbias=1e-5, dW=1e-5, mom=1e-5, W=3e-6, gain=1e-6, bias=1e-5)
    for k, t in tol.items():
        e = rel_fro(host64(s[k]), ref[k])
        assert e <= t, f"{k}: {e:.2e} > {t:.0e}"
    assert torch.equal(s["W_lp"], s["W"].to(dtype))


def test_captured_step_replays_match_eager(dev):
    eager, graphed = make(dev, torch.bfloat16), make(dev, torch.bfloat16)
    for s in (eager, graphed):
        step(s, 1, torch.bfloat16)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        step(graphed, 2, torch.bfloat16)
    for _ in range(3):
        step(eager, 2, torch.bfloat16)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for k in ("y", "dx", "dgain", "dbias", "dW", "W", "W_lp", "mom", "gain", "bias", "W_sumsq", "p_sumsq"):
            assert torch.equal(eager[k], graphed[k]), k


OUT = ("y", "dx", "dx_lp", "dgain", "dbias", "dW", "W", "W_lp", "mom", "gain", "bias", "W_sumsq", "p_sumsq", "clip")


def test_two_threads_two_streams(dev):
    """Two host threads, each on its own stream with its own buffers, as if each were alone."""
    ref = [make(dev, torch.bfloat16, seed) for seed in (1, 2)]
    for s in ref:
        for k in (1, 2, 3):
            step(s, k, torch.bfloat16)
    got = [make(dev, torch.bfloat16, seed) for seed in (1, 2)]
    torch.cuda.synchronize()
    errors = []

    def run(s):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for k in (1, 2, 3):
                    step(s, k, torch.bfloat16)
            st.synchronize()
        except Exception as e:  # pragma: no cover - reported below
            errors.append(e)

    threads = [threading.Thread(target=run, args=(s,)) for s in got]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for r, s in zip(ref, got):
        for k in OUT:
            assert torch.equal(r[k], s[k]), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_large_tiles_captured_and_replayed(dev, dtype):
    """The Muon step on sizes that take the large tiles, whole and in quarters, and on small
    ones beside them: eager twice and captured, the same bits."""
    shapes = [(2048, 2560)] * 4 + [(2560, 2048)] * 4 + [(72, 200), (1288, 1544)]
    g = torch.Generator(device=dev)

    def state():
        g.manual_seed(5)
        r = lambda s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
        return dict(grad=[r(x) for x in shapes], W=[0.02 * r(x) for x in shapes], state=[r(x) for x in shapes],
                    W_lp=[torch.empty(*x, device=dev, dtype=dtype) for x in shapes],
                    sumsq=torch.ones(len(shapes), device=dev, dtype=torch.float64),
                    ws=api.workspace(api.fpo_muon_update_workspace(shapes, dtype), dev))

    def run(s):
        api.fpo_muon_update(api.MuonConfig(lr=1e-2, clip_frac=0.0, step=2), s["grad"], s["W"], s["state"],
                            W_sumsq=s["sumsq"], W_lp=s["W_lp"], dtype=dtype, ws=s["ws"])

    eager, again, graphed = state(), state(), state()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        run(graphed)
    for _ in range(3):
        run(eager)
        run(again)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for s in (again, graphed):
            assert torch.equal(eager["sumsq"], s["sumsq"])
            for k in ("W", "state", "W_lp"):
                assert all(torch.equal(a, b) for a, b in zip(eager[k], s[k])), k
    for W, q, lp in zip(eager["W"], eager["sumsq"].tolist(), eager["W_lp"]):
        assert torch.isfinite(W).all() and torch.equal(lp, W.to(dtype))
        assert abs(q / W.double().square().sum().item() - 1) < 1e-12
