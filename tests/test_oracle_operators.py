"""Pins of oracle/operators.py: the orthogonalisation against the singular value
decomposition, the Muon step against its parts, layer norm and its VJP against
torch's autograd and against differences (CPU)."""
import numpy as np
import pytest
import torch

from oracle import operators as P

RNG = np.random.default_rng


def poly(s, steps, coefs):
    for a, b, c in coefs if not isinstance(coefs[0], float) else [coefs] * steps:
        s = a * s + b * s ** 3 + c * s ** 5
    return s


@pytest.mark.parametrize("shape", [(8, 8), (16, 40), (40, 16), (1, 24)])
@pytest.mark.parametrize("coefs", [P.MUON_COEF, (1.5, -0.5, 0.0), [(4.0, -7.0, 4.0), (3.4445, -4.7750, 2.0315)]])
def test_newton_schulz_maps_singular_values(shape, coefs):
    """O has M's singular vectors and the polynomial's values, in either orientation."""
    steps = 5 if isinstance(coefs, tuple) else 2
    M = RNG(0).normal(size=shape)
    U, s, Vt = np.linalg.svd(M, full_matrices=False)
    want = (U * poly(s / np.linalg.norm(M), steps, coefs)) @ Vt
    got = P.newton_schulz(M, steps, coefs, eps=0.0)
    assert np.abs(got - want).max() < 1e-12


def test_newton_schulz_converges_to_the_polar_factor():
    M = RNG(1).normal(size=(12, 30))
    U, s, Vt = np.linalg.svd(M, full_matrices=False)
    O = P.newton_schulz(M, 40, (1.5, -0.5, 0.0))
    assert np.abs(O - U @ Vt).max() < 1e-12
    assert np.abs(P.newton_schulz(M, 5) @ P.newton_schulz(M, 5).T - np.eye(12)).max() < 0.6  # Muon's coefficients


def test_newton_schulz_zero_and_scale():
    assert not P.newton_schulz(np.zeros((4, 8)), eps=0.0).any()
    M = RNG(2).normal(size=(6, 10))
    assert np.abs(P.newton_schulz(1e6 * M, eps=0.0) - P.newton_schulz(M, eps=0.0)).max() < 1e-12


def test_rounded_newton_schulz_error_follows_the_type():
    M = RNG(3).normal(size=(48, 130))
    E = P.newton_schulz(M)

    def err(t):
        return np.linalg.norm(P.rounded_newton_schulz(M, dtype=t) - E) / np.linalg.norm(E)

    assert 1e-4 < err(np.float16) < 1e-2 and 1e-8 < err(np.float32) < 2e-6


def test_muon_parts():
    rng = RNG(4)
    W, g, b = rng.normal(size=(3, 8, 24))
    O = P.newton_schulz(g + 0.9 * (0.9 * b + g))
    W1, b1, k, _ = P.muon(W, g, b, lr=0.1, momentum=0.9, weight_decay=0.02, scale="rms", step=3)
    assert k == 1.0 and np.allclose(b1, 0.9 * b + g)
    assert np.allclose(W1, W * (1 - 0.1 * 0.02) - 0.1 * 0.2 * np.sqrt(24) * O)
    W1, b1, _, _ = P.muon(W.T, g.T, None, lr=0.1, momentum=0.0, scale="spectral")
    assert np.allclose(W1, W.T - 0.1 * np.sqrt(3) * P.newton_schulz(g).T)
    for clip, limit in (("update", None), ("gradient", None)):
        W1, _, k, u = P.muon(W, g, b, lr=0.5, momentum=0.9, step=2, clip_frac=0.01, clip=clip)
        assert k < 1.0
        if clip == "update":
            assert np.isclose(np.linalg.norm(W1 - W), 0.01 * np.linalg.norm(W))
    W1, b1, _, u = P.muon(W, g, b, lr=0.5, momentum=0.9, nesterov=False, step=1)
    assert np.array_equal(b1, g) and np.array_equal(u, g)


@pytest.mark.parametrize("affine", [True, False])
def test_layernorm_and_vjp_against_autograd(affine):
    rng = RNG(5)
    x = torch.tensor(rng.normal(size=(7, 24)) * 3 + 2, requires_grad=True)
    gain = torch.tensor(rng.normal(size=24), requires_grad=True) if affine else None
    bias = torch.tensor(rng.normal(size=24), requires_grad=True) if affine else None
    dy = torch.tensor(rng.normal(size=(7, 24)))
    y = torch.nn.functional.layer_norm(x, (24,), gain, bias, 1e-5)
    y.backward(dy)
    n = lambda t: None if t is None else t.detach().numpy()  # noqa: E731
    assert np.allclose(P.layernorm(n(x), n(gain), n(bias))[0], n(y), atol=1e-13)
    dx, dgain, dbias = P.layernorm_vjp(n(x), n(gain), dy.numpy())
    assert np.allclose(dx, x.grad.numpy(), atol=1e-13)
    if affine:
        assert np.allclose(dgain, gain.grad.numpy()) and np.allclose(dbias, bias.grad.numpy())


def test_layernorm_vjp_against_differences():
    rng = RNG(6)
    x, dy, gain = rng.normal(size=(3, 16)), rng.normal(size=(3, 16)), rng.normal(size=16)
    dx, dgain, _ = P.layernorm_vjp(x, gain, dy)
    h = 1e-6
    for t, j in ((0, 0), (1, 7), (2, 15)):
        e = np.zeros_like(x)
        e[t, j] = h
        d = ((P.layernorm(x + e, gain)[0] - P.layernorm(x - e, gain)[0]) * dy).sum() / (2 * h)
        assert abs(d - dx[t, j]) < 1e-8
        e = np.zeros(16)
        e[j] = h
        d = ((P.layernorm(x, gain + e)[0] - P.layernorm(x, gain - e)[0]) * dy).sum() / (2 * h)
        assert abs(d - dgain[j]) < 1e-8


def test_layernorm_vjp_floor():
    """Where sigma is under the floor, dx is the exact VJP of a norm whose epsilon lifts
    sigma to it; elsewhere the floor changes nothing."""
    rng = RNG(7)
    x = rng.normal(size=(2, 32)) * np.array([[0.01], [2.0]])
    dy, gain = rng.normal(size=(2, 32)), rng.normal(size=32)
    dx, dgain, _ = P.layernorm_vjp(x, gain, dy, min_std=0.5)
    exact, g0, _ = P.layernorm_vjp(x, gain, dy)
    assert np.array_equal(dx[1], exact[1]) and np.array_equal(dgain, g0)
    lifted = P.layernorm_vjp(x[:1], gain, dy[:1], eps=0.25 - x[0].var())[0]
    assert np.allclose(dx[0], lifted[0])
