"""Float64 CPU oracle of the orthogonalisation, the Muon step and layer norm
(test infrastructure only; shares no code with the library).

newton_schulz and muon are written from their definitions; layernorm and
layernorm_vjp from the definition of the norm and its Jacobian, with the floor
on sigma that the RMSNorm VJPs have on rho. rounded_newton_schulz is the same
iteration with every matrix that it stores rounded to a narrower type: what one
rounding a matrix costs at the given input, against which errors are judged.
"""
from __future__ import annotations

import math

import numpy as np

MUON_COEF = (3.4445, -4.7750, 2.0315)


def _per_step(coefs, steps):
    if coefs is None:
        coefs = MUON_COEF
    return [tuple(coefs)] * steps if isinstance(coefs[0], (int, float)) else [tuple(c) for c in coefs]


def newton_schulz(M, steps=5, coefs=None, eps=1e-7):
    """X = M / (||M||_F + eps), then X <- a X + b (X X^T) X + c (X X^T)^2 X at every step."""
    X = np.asarray(M, dtype=np.float64)
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    norm = math.sqrt(float((X * X).sum())) + eps
    X = X / norm if norm > 0 else np.zeros_like(X)
    for a, b, c in _per_step(coefs, steps):
        A = X @ X.T
        X = a * X + b * (A @ X) + c * (A @ (A @ X))
    return X.T if tall else X


def rounded_newton_schulz(M, steps=5, coefs=None, eps=1e-7, dtype=np.float16, groups=None,
                          accumulate=False):
    """newton_schulz with X, X X^T and a I + b X X^T + c (X X^T)^2 rounded to `dtype`
    wherever they are stored (float16 with a power of two that keeps it in range),
    products and sums exact, or with `accumulate` the sums of products in float32, one
    after the other. groups: numbers of steps for which X X^T is formed once
    and carried on as B A B (rounded, B A too), X being multiplied by the rounded
    product of their B; one step each if None."""
    X = np.asarray(M, dtype=np.float64)
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    scale = 512.0 if dtype == np.float16 else 1.0

    def r(v, s=scale):
        return (v * s).astype(dtype).astype(np.float64) / s

    def mm(x, y):
        if not accumulate:
            return x @ y
        acc = np.zeros((x.shape[0], y.shape[1]), np.float32)
        for k in range(x.shape[1]):
            acc = (acc + np.outer(x[:, k], y[k])).astype(np.float32)
        return acc.astype(np.float64)

    norm = math.sqrt(float((X * X).sum())) + eps
    X = X / norm if norm > 0 else np.zeros_like(X)
    eye = np.eye(X.shape[0])
    per_step = _per_step(coefs, steps)
    at = 0
    for count in groups or [1] * steps:
        X = r(X, 8 * scale)
        A, Q = r(mm(X, X.T)), None
        for j in range(count):
            a, b, c = per_step[at + j]
            B = r(a * eye + b * A + c * mm(A, A))
            Q = B if Q is None else r(mm(B, Q))
            if j + 1 < count:
                A = r(mm(r(mm(B, A)), B))
        X = mm(Q, X)
        at += count
    return X.T if tall else X


def muon_scale(kind, rows, cols):
    """'none', 'spectral' or 'rms'."""
    return {"none": 1.0, "spectral": math.sqrt(max(1.0, rows / cols)), "rms": 0.2 * math.sqrt(max(rows, cols))}[kind]


def muon(W, grad, buf, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale="rms", step=1, clip_frac=0.0,
         clip="gradient", steps=5, coefs=None, eps=1e-7, orthogonal=None):
    """One step: (W', b', clip factor, u). `orthogonal`: O, if it is already known."""
    W, g = np.asarray(W, np.float64), np.asarray(grad, np.float64)

    def factor(limit, size):
        return 1.0 if clip_frac <= 0 or size == 0 else min(1.0, clip_frac * limit / size)

    k = factor(np.linalg.norm(W), np.linalg.norm(g)) if clip == "gradient" else 1.0
    g = k * g
    b = g if step == 1 or buf is None else momentum * np.asarray(buf, np.float64) + g
    u = g + momentum * b if nesterov and buf is not None else b
    O = newton_schulz(u, steps, coefs, eps) if orthogonal is None else np.asarray(orthogonal, np.float64)
    delta = -lr * weight_decay * W - lr * muon_scale(scale, *W.shape) * O
    if clip == "update":
        k = factor(np.linalg.norm(W), np.linalg.norm(delta))
        delta = k * delta
    return W + delta, b, k, u


def layernorm(x, gain=None, bias=None, eps=1e-5):
    """(y, mean, 1 / sigma) of each row."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1, keepdims=True)
    sigma = np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mean) / sigma
    if gain is not None:
        y = y * np.asarray(gain, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, mean[:, 0], 1.0 / sigma[:, 0]


def layernorm_vjp(x, gain, dy, eps=1e-5, min_std=0.0):
    """(dx, dgain, dbias); sigma is floored at min_std in dx only."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    xc = x - x.mean(1, keepdims=True)
    sigma = np.sqrt((xc ** 2).mean(1, keepdims=True) + eps)
    dgain, dbias = (dy * xc / sigma).sum(0), dy.sum(0)
    sigma = np.maximum(sigma, min_std)
    xh = xc / sigma
    v = dy if gain is None else dy * np.asarray(gain, np.float64)
    dx = (v - v.mean(1, keepdims=True) - xh * (v * xh).mean(1, keepdims=True)) / sigma
    return dx, dgain, dbias
