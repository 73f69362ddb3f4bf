"""fpo_layernorm_vjp where a workgroup sums the gradients of gain and bias over several rows:
long rows, which share the fewest workgroups, and the few rows that one workgroup keeps.

Tolerance of the sums over rows, relative to the sum of the terms' magnitudes: a lane adds
every (n slots)-th row in float32, the workgroup's slots are added in float32, the n
workgroups in float64, rounded once; u = 2^-24 an addition, and 4 u for a term itself and
the result. n is read from the workspace (two rows of d floats a workgroup; none: one), the
slots from the row's length: rows of up to 128, 256 and 1024 elements have 16, 32 and 64
lanes of a workgroup's 256, longer ones all. The rest is bounded as in
test_parity_layernorm."""
import os

import numpy as np
import pytest
import torch

from paper_2608_14563_amd import _lib as L
from paper_2608_14563_amd import api
from tests._util import host64
from tests.test_parity_layernorm import check, forward_tol, rows, vjp_tol

BF, F32 = torch.bfloat16, torch.float32


def layout(T, d):
    """(workgroups, rows at once in each)."""
    need = api.fpo_layernorm_vjp_workspace(T, d)
    slots = 16 if d <= 128 else 8 if d <= 256 else 4 if d <= 512 or (d <= 1024 and T >= 1024) else 1
    return (need // (8 * d) if need else 1), slots


LONG = [(2101, 4104), (1301, 8192), (1001, 8200), (600, 16384), (523, 16392)]
FEW = [(64, 128), (65, 128), (16, 512), (17, 512), (2, 4096), (3, 4096), (2, 8192), (3, 8192), (1, 16384), (2, 16384)]


@pytest.fixture(scope="module")
def built():
    if not os.path.exists(L.LIB_PATH):
        pytest.fail("libfpo.so is not built (run __graft_entry__.build())")


@pytest.mark.parametrize("T,d", LONG)
def test_long_rows_share_256_workgroups(built, T, d):
    assert layout(T, d) == (256, 1) and T > 2 * 256


@pytest.mark.parametrize("T,d", FEW)
def test_few_rows_are_one_workgroups(built, T, d):
    n, slots = layout(T, d)
    groups = -(-T // slots)
    assert n == (1 if groups <= {16: 4, 8: 4, 4: 4, 1: 2}[slots] and (d <= 8192 or T == 1) else groups)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dy_dtype", [(BF, F32), (F32, F32)], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", LONG + FEW)
def test_parameter_gradients(dev, T, d, dtype, dy_dtype):
    n, slots = layout(T, d)
    x, gain = rows(T, d, dev, dtype, seed=T), rows(1, d, dev, dtype, seed=1)[0]
    dy = 0.02 * rows(T, d, dev, F32, seed=2)
    nan = lambda s, t: torch.full(s, float("nan"), dtype=t, device=dev)  # noqa: E731
    out = dict(dx=nan((T, d), F32), dx_lp=nan((T, d), dtype), dgain=nan((d,), F32), dbias=nan((d,), F32))
    api.fpo_layernorm_vjp(x, gain, dy.to(dy_dtype), **out)
    added = -(-T // (n * slots)) + slots
    dx, dg, db, tdx, tdg, tdb = vjp_tol(host64(x), host64(gain), host64(dy), 1e-5, 0.0, added)
    check("dx", out["dx"], dx, tdx, F32)
    check("dx_lp", out["dx_lp"], dx, tdx, dtype)
    check("dgain", out["dgain"], dg, tdg, F32)
    check("dbias", out["dbias"], db, tdb, F32)
    assert np.isfinite(host64(out["dgain"])).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 1032, 4104])
@pytest.mark.parametrize("scale,eps", [(1e-14, 0.0), (1e-14, 1e-30), (None, 0.0), (None, 1e-5)], ids=["small", "small-eps", "large", "large-eps"])
def test_range_of_the_statistics(dev, d, scale, eps):
    """Deviations from 1e-15 (here ten times that, and a row of 1e-15) up to entries of 1e18 /
    sqrt(d): of normal values none is more than 6 deviations from the mean."""
    T = 9
    x = rows(T, d, dev, F32, seed=d)
    assert x.abs().max() < 6
    x.mul_(1e18 / (6 * d ** 0.5) if scale is None else scale)
    if scale is not None:
        x[3] *= 0.1
    gain, dy = rows(1, d, dev, F32, seed=1)[0], 0.02 * rows(T, d, dev, F32, seed=2)
    y, dx, dgain = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device=dev)
    api.fpo_layernorm(x, gain, None, y, eps=eps)
    api.fpo_layernorm_vjp(x, gain, dy, dx=dx, dgain=dgain, eps=eps)
    want, _, _, tol = forward_tol(host64(x), host64(gain), None, eps)
    check("y", y, want, tol, F32)
    n, slots = layout(T, d)
    wx, wg, _, tdx, tdg, _ = vjp_tol(host64(x), host64(gain), host64(dy), eps, 0.0, -(-T // (n * slots)) + slots)
    check("dx", dx, wx, tdx, F32)
    check("dgain", dgain, wg, tdg, F32)
