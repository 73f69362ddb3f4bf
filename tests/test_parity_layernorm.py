"""fpo_layernorm and fpo_layernorm_vjp on the GPU against oracle/operators.py.

Tolerances, entry by entry. u = 2^-24. A sum over a row goes through at most 4 chunks
of 8 elements a lane and 10 stages between lanes, fewer than 32 roundings: mean is
off by 32 u mean|x| at most, sigma relatively by 32 u (half of that, and the root and
the quotient), hence y by 64 u ((|x| + mean|x|) / sigma |gain|) + 4 u (|y| + |bias|).
dx adds two row sums with as many roundings each; the parameter gradients a sum over
tokens, in float32 over the rows of one workgroup (at least 512 share T, and up to 16
rows at once are added at the end) and in float64 between them. Rows of more than 16384 elements add d / 8192 more roundings a lane. bf16
results add half a step, 2^-8 relative."""
import numpy as np
import pytest
import torch

from oracle import operators as P
from paper_2608_14563_amd import api
from tests._util import host64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def rows(T, d, dev, dtype, seed=0, kind="normal"):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(T, d)).astype(np.float32)
    if kind == "offset":   # a mean a thousand times the deviation
        x = 1000 + x
    elif kind == "spread":  # nearly constant rows, huge rows, one outlier
        x = x * np.exp(rng.normal(size=(T, 1)) * 3)
        x[:, 0] *= 100
    elif kind == "constant":
        x[:] = 3.0
    return torch.from_numpy(x.astype(np.float32)).to(dev).to(dtype)


def n_round(d):
    return 32 + d // 8192


def check(name, got, want, tol, dtype):
    tol = tol + (2.0 ** -8 * np.abs(want) if dtype == BF else 0) + 1e-37
    off = np.abs(host64(got) - want) / tol
    assert not (off > 1).any() and np.isfinite(host64(got)).all(), f"{name}: {np.nanmax(off):.2f} times the tolerance"


def forward_tol(x, gain, bias, eps):
    y, mean, rstd = P.layernorm(x, gain, bias, eps)
    d = x.shape[1]
    g = 1 if gain is None else np.abs(gain)
    t = 2 * n_round(d) * U * (np.abs(x) + np.abs(x).mean(1, keepdims=True)) * rstd[:, None] * g + 4 * U * (
        np.abs(y) + (0 if bias is None else np.abs(bias)))
    return y, mean, rstd, t


def vjp_tol(x, gain, dy, eps, min_std, T_block):
    dx, dg, db = P.layernorm_vjp(x, gain, dy, eps, min_std)
    d = x.shape[1]
    n = n_round(d) * U
    xc = x - x.mean(1, keepdims=True)
    sig = np.sqrt((xc ** 2).mean(1, keepdims=True) + eps)
    inv = 1 / np.maximum(sig, min_std)
    v = dy if gain is None else dy * gain
    av, size = np.abs(v), np.abs(x) + np.abs(x).mean(1, keepdims=True)
    xh, axh = np.abs(xc) * inv, size * inv
    m1, m2 = av.mean(1, keepdims=True), (av * axh).mean(1, keepdims=True)
    tdx = 4 * n * (av + m1 + (axh + xh) * m2 + axh * (av * xh).mean(1, keepdims=True)) * inv
    rows_ = (T_block + 4) * U
    tdg = 2 * n * (np.abs(dy) * size / sig).sum(0) + rows_ * np.abs(dy * xc / sig).sum(0)
    return dx, dg, db, tdx, tdg, rows_ * np.abs(dy).sum(0)


CASES = [(1, 8), (1, 4096), (3, 64), (5, 72), (7, 512), (9, 520), (33, 1024), (17, 1032), (611, 2048), (13, 2056),
         (40, 4096), (6, 4104), (11, 8192), (5, 8200), (3, 16384), (4, 16392), (2, 65536),
         (1, 128), (300, 128), (999, 136), (701, 256), (1201, 264), (20001, 64), (9001, 248)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", CASES)
def test_forward(dev, T, d, dtype):
    x = rows(T, d, dev, dtype, seed=T + d)
    gain, bias = (rows(1, d, dev, dtype, seed=k)[0] for k in (1, 2))
    y = torch.full((T, d), float("nan"), dtype=dtype, device=dev)
    mean, rstd = torch.empty(T, device=dev), torch.empty(T, device=dev)
    api.fpo_layernorm(x, gain, bias, y, mean=mean, rstd=rstd)
    xs = host64(x)
    want, wm, wr, tol = forward_tol(xs, host64(gain), host64(bias), 1e-5)
    check("y", y, want, tol, dtype)
    check("mean", mean, wm, n_round(d) * U * np.abs(xs).mean(1), F32)
    check("rstd", rstd, wr, n_round(d) * U * wr * (1 + np.abs(xs).mean(1) * wr * U), F32)


@pytest.mark.parametrize("kind", ["offset", "spread", "constant"])
@pytest.mark.parametrize("affine", ["both", "gain", "none"])
def test_forward_values(dev, kind, affine):
    T, d = 37, 1544
    x = rows(T, d, dev, F32, seed=3, kind=kind)
    gain = rows(1, d, dev, F32, seed=1)[0] if affine != "none" else None
    bias = rows(1, d, dev, F32, seed=2)[0] if affine == "both" else None
    y = torch.empty_like(x)
    api.fpo_layernorm(x, gain, bias, y)
    xs, h = host64(x), lambda t: None if t is None else host64(t)  # noqa: E731
    want, _, rstd, tol = forward_tol(xs, h(gain), h(bias), 1e-5)
    # with a large mean sigma is off by the error of the mean too: (err / sigma)^2 / 2 relative, far below the rest
    check("y", y, want, tol, F32)


def run_vjp(dev, T, d, dtype, dy_dtype, min_std=0.0, kind="normal", seed=0, scale=None):
    x = rows(T, d, dev, dtype, seed=seed + T + d, kind=kind)
    if scale is not None:
        x = (x.float() * torch.tensor(scale, device=dev)[:, None]).to(dtype)
    gain = rows(1, d, dev, dtype, seed=1)[0]
    dy = (0.02 * rows(T, d, dev, F32, seed=9 + T)).to(dy_dtype)
    nan = lambda s, t: torch.full(s, float("nan"), dtype=t, device=dev)  # noqa: E731
    out = dict(dx=nan((T, d), F32), dx_lp=nan((T, d), dtype), dgain=nan((d,), F32), dbias=nan((d,), F32))
    api.fpo_layernorm_vjp(x, gain, dy, min_std=min_std, **out)
    block = -(-T // 512) + 16
    dx, dg, db, tdx, tdg, tdb = vjp_tol(host64(x), host64(gain), host64(dy), 1e-5, min_std, block)
    check("dx", out["dx"], dx, tdx, F32)
    check("dx_lp", out["dx_lp"], dx, tdx, dtype)
    check("dgain", out["dgain"], dg, tdg, F32)
    check("dbias", out["dbias"], db, tdb, F32)
    return x, gain, dy, out


@pytest.mark.parametrize("dtype,dy", [(BF, F32), (BF, BF), (F32, F32), (F32, BF)], ids=["bf16-f32", "bf16", "f32", "f32-bf16"])
@pytest.mark.parametrize("T,d", CASES)
def test_vjp(dev, T, d, dtype, dy):
    run_vjp(dev, T, d, dtype, dy)


def test_vjp_many_rows(dev):
    """More rows than workgroups, one row or several at once in each."""
    for T, d in ((9001, 72), (5003, 256), (2600, 2056)):
        run_vjp(dev, T, d, BF, F32)


def test_offsets_past_32_bits(dev):
    """More than 2^31 elements; the first and last rows against the oracle, the parameter
    gradients against float64 sums over all of them."""
    T, d = (1 << 19) + 77, 4104
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    x = torch.empty(T, d, device=dev, dtype=BF).normal_(generator=g)
    dy = torch.empty(T, d, device=dev, dtype=BF).normal_(generator=g)
    gain = rows(1, d, dev, BF, 4)[0]
    y, dx_lp = torch.empty_like(x), torch.empty_like(x)
    dgain, dbias = torch.empty(d, device=dev), torch.empty(d, device=dev)
    api.fpo_layernorm(x, gain, None, y)
    api.fpo_layernorm_vjp(x, gain, dy, dx_lp=dx_lp, dgain=dgain, dbias=dbias)
    for part in (slice(0, 3), slice(T // 2, T // 2 + 3), slice(T - 3, T)):
        xs, ds = host64(x[part]), host64(dy[part])
        Y, _, _, ty = forward_tol(xs, host64(gain), None, 1e-5)
        check("y", y[part], Y, ty, BF)
        dx, _, _, tdx, _, _ = vjp_tol(xs, host64(gain), ds, 1e-5, 0.0, 3)
        check("dx_lp", dx_lp[part], dx, tdx, BF)
    wg, wb, ag, ab, size = [torch.zeros(d, device=dev, dtype=torch.float64) for _ in range(5)]
    for i in range(0, T, 1 << 15):
        xs, ds = x[i:i + (1 << 15)].double(), dy[i:i + (1 << 15)].double()
        xc = xs - xs.mean(1, keepdim=True)
        rstd = 1 / (xc.square().mean(1, keepdim=True) + 1e-5).sqrt()
        wg += (ds * xc * rstd).sum(0)
        wb += ds.sum(0)
        ag += (ds * xc * rstd).abs().sum(0)
        ab += ds.abs().sum(0)
        size += (ds.abs() * (xs.abs() + xs.abs().mean(1, keepdim=True)) * rstd).sum(0)
    r = (T // 256 + 5) * U  # (rows of this length run on 256 workgroups at least)
    assert ((dgain - wg).abs() <= r * ag + 2 * n_round(d) * U * size).all()
    assert ((dbias - wb).abs() <= r * ab).all()


def test_vjp_floor(dev):
    """Rows under, around and over the floor."""
    T, d = 64, 1032
    run_vjp(dev, T, d, F32, F32, min_std=0.5, scale=np.geomspace(1e-3, 10, T).astype(np.float32))
    run_vjp(dev, 5, 64, F32, F32, kind="constant", min_std=0.25)


@pytest.mark.parametrize("keep", [("dx",), ("dx_lp",), ("dgain",), ("dbias",), ("dgain", "dbias"), ("dx", "dbias")],
                         ids="-".join)
@pytest.mark.parametrize("T,d", [(1, 64), (300, 520), (70, 2056), (3, 16392)])
def test_vjp_each_output_alone(dev, T, d, keep):
    """Outputs left out change nothing in the others."""
    x, gain, dy, out = run_vjp(dev, T, d, BF, F32)
    some = {k: torch.full_like(out[k], float("nan")) for k in keep}
    ws = api.workspace(api.fpo_layernorm_vjp_workspace(T, d), dev).fill_(255)
    api.fpo_layernorm_vjp(x, gain, dy, ws=ws, **some)
    for k in keep:
        assert torch.equal(some[k], out[k]), k


def test_without_gain_and_bias(dev):
    x = rows(19, 264, dev, F32)
    dy = rows(19, 264, dev, F32, seed=4)
    y, y1 = torch.empty_like(x), torch.empty_like(x)
    one, zero = torch.ones(264, device=dev), torch.zeros(264, device=dev)
    api.fpo_layernorm(x, None, None, y)
    api.fpo_layernorm(x, one, zero, y1)
    assert torch.equal(y, y1)
    a, b = torch.empty_like(x), torch.empty_like(x)
    api.fpo_layernorm_vjp(x, None, dy, dx=a)
    api.fpo_layernorm_vjp(x, one, dy, dx=b)
    assert torch.equal(a, b)


def test_bad_row_keeps_to_itself(dev):
    """A row with a NaN or an infinity: the other rows are as without it; the parameter
    gradients, sums over all rows, are not finite."""
    for d in (72, 2056):
        x = rows(9, d, dev, F32)
        gain, bias, dy = (rows(k, d, dev, F32, seed=5 + k) for k in (1, 1, 9))
        y, dx = torch.empty_like(x), torch.empty_like(x)
        api.fpo_layernorm(x, gain[0], bias[0], y)
        api.fpo_layernorm_vjp(x, gain[0], dy, dx=dx)
        for bad in (float("nan"), float("inf"), -float("inf")):
            z = x.clone()
            z[4, 3] = bad
            y1, dx1, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device=dev)
            api.fpo_layernorm(z, gain[0], bias[0], y1)
            api.fpo_layernorm_vjp(z, gain[0], dy, dx=dx1, dgain=dg)
            keep = [t for t in range(9) if t != 4]
            assert torch.equal(y1[keep], y[keep]) and torch.equal(dx1[keep], dx[keep])
            assert not torch.isfinite(y1[4]).any() and not torch.isfinite(dx1[4]).any()
            assert not torch.isfinite(dg).any()


def test_leaves_what_surrounds_it(dev):
    T, d = 7, 2056
    buf = torch.full((T * d + 256,), 7.0, device=dev)
    out = buf[128:128 + T * d].view(T, d)
    x, dy = rows(T, d, dev, F32), rows(T, d, dev, F32, seed=2)
    small = torch.full((d + 64,), 7.0, device=dev)
    api.fpo_layernorm(x, None, None, out)
    assert (buf[:128] == 7).all() and (buf[128 + T * d:] == 7).all()
    api.fpo_layernorm_vjp(x, None, dy, dx=out, dgain=small[32:32 + d])
    assert (buf[:128] == 7).all() and (buf[128 + T * d:] == 7).all()
    assert (small[:32] == 7).all() and (small[32 + d:] == 7).all()


def test_graph_replays_match_eager(dev):
    T, d = 600, 1032
    x, dy, gain = rows(T, d, dev, BF), rows(T, d, dev, F32, seed=2), rows(1, d, dev, BF, seed=3)[0]
    ws = api.workspace(api.fpo_layernorm_vjp_workspace(T, d), dev)

    def outs():
        return dict(y=torch.empty_like(x), dx=torch.empty(T, d, device=dev), dx_lp=torch.empty_like(x),
                    dgain=torch.empty(d, device=dev), dbias=torch.empty(d, device=dev))

    def go(o, ws):
        api.fpo_layernorm(x, gain, gain, o["y"])
        api.fpo_layernorm_vjp(x, gain, dy, **{k: o[k] for k in ("dx", "dx_lp", "dgain", "dbias")}, ws=ws)

    eager, graphed = outs(), outs()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        go(graphed, ws)
    for k in range(3):
        x.mul_(0.5).add_(k)
        go(eager, ws)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(eager[n], graphed[n]), n
