"""The final layer norm of a model without a bias there, from two calls: fpo_output_error on
the centred hidden states x - mean x, whose RMSNorm is the layer norm, for the error g_pre
behind the norm, and fpo_layernorm_vjp of it, with the gain's gradient.

Tolerances: the output error's own (1e-5, bf16 2e-2 relative Frobenius, cosine 0.9999), which
the VJP, linear in its error, carries on; dgain sums over the tokens with them."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import operators as P
from paper_2608_14563_amd import api
from tests._util import assert_close, host64

T, D, V, EPS = 200, 136, 1000, 1e-5


def inputs():
    rng = np.random.default_rng(5)
    x = rng.normal(size=(T, D)) * np.exp(0.5 * rng.normal(size=(T, 1))) + 0.7
    xc = x - x.mean(1, keepdims=True)
    return xc, 1 + 0.1 * rng.normal(size=D), 0.1 * rng.normal(size=(V, D)), rng.integers(0, V, T).astype(np.int32)


def expected(xc, gain, W, y, min_std):
    """In float64, from the layer norm's definition."""
    z = P.layernorm(xc, gain, None, EPS)[0] @ W.T
    e = np.exp(z - z.max(1, keepdims=True))
    e /= e.sum(1, keepdims=True)
    e[np.arange(T), y] -= 1
    g = e @ W
    return g, *P.layernorm_vjp(xc, gain, g, EPS, min_std)[:2]


def test_rmsnorm_of_centred_states_is_the_layer_norm():
    """g_pre and its VJP are the gradients of the cross entropy behind a layer norm (autograd)."""
    xc, gain, W, y = inputs()
    g = O.output_error(xc, gain, W, y, eps=EPS)["g_pre"]
    dx, dgain, _ = P.layernorm_vjp(xc, gain, g, EPS)
    x, w = torch.from_numpy(xc + 0.7).requires_grad_(), torch.from_numpy(gain).requires_grad_()
    z = torch.nn.functional.layer_norm(x, (D,), w, None, EPS) @ torch.from_numpy(W).t()
    torch.nn.functional.cross_entropy(z, torch.from_numpy(y).long(), reduction="sum").backward()
    np.testing.assert_allclose(dx, x.grad.numpy(), rtol=1e-9, atol=1e-11)
    np.testing.assert_allclose(dgain, w.grad.numpy(), rtol=1e-9, atol=1e-11)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("min_std", [0.0, 0.5])
def test_layer_norm_behind_the_output_error(dev, dtype, min_std):
    lp = torch.bfloat16 if dtype == "bf16" else torch.float32
    xc, gain, W, y = inputs()
    h, g, w = (torch.from_numpy(a).to(dev).to(lp) for a in (xc, gain, W))
    pre, out, dx, dgain = (torch.empty(s, device=dev) for s in ((T, D), (T, D), (T, D), (D,)))
    api.fpo_output_error(h, g, w, torch.from_numpy(y).to(dev), out, g_pre=pre, eps=EPS)
    api.fpo_layernorm_vjp(h, g, pre, dx=dx, dgain=dgain, eps=EPS, min_std=min_std)
    for name, got, want in zip(("g_pre", "dx", "dgain"), (pre, dx, dgain),
                               expected(host64(h), host64(g), host64(w), y, min_std)):
        assert_close(name, host64(got), want, dtype)
