"""Calls whose written buffers share memory with another buffer of the call: refused
before anything is launched (CPU). Addresses are never dereferenced."""
import ctypes as C
import os

import pytest

from paper_2608_14563_amd import _lib as L

ROWS, COLS = 64, 128
SIZE = ROWS * COLS * 4       # of a float32 matrix
BASE, WS = 1 << 20, 1 << 40  # matrices from BASE on, the workspace far behind them


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.fail("libfpo.so is not built (run __graft_entry__.build())")
    return L.load()


def i64(*v):
    return (C.c_int64 * len(v))(*v)


def ptrs(*v):
    return (C.c_void_p * len(v))(*v)


# --------------------------------------------------------------------- the Muon step
def muon(lib, dtype=L.FPO_BF16, momentum=0.9, ws=WS, **over):
    """Two matrices whose buffers follow each other without a gap; over: name=(matrix, address)."""
    bufs, at = {}, BASE
    for k in ("grad", "W_master", "state1", "W_lp"):
        bufs[k] = []
        for _ in range(2):
            bufs[k].append(at)
            at += SIZE // 2 if k == "W_lp" and dtype == L.FPO_BF16 else SIZE
    for k, (m, address) in over.items():
        bufs[k][m] = address
    o = L.Muon(L.NsDesc(dtype, 5, 1e-7, None), 1e-3, momentum, 0.01, 0.0, 2, 1, 2, 0)
    u = L.UpdateBufs(ptrs(*bufs["W_master"]), ptrs(*bufs["W_lp"]), ptrs(*bufs["state1"]), None, None, None)
    status = lib.fpo_muon_update(C.byref(o), 2, i64(ROWS, ROWS), i64(COLS, COLS), ptrs(*bufs["grad"]), None, C.byref(u),
                                 ws, 1 << 30, None)
    return status, lib.fpo_last_error().decode()


GRAD, W, STATE, LP = (BASE + 2 * k * SIZE for k in range(4))


@pytest.mark.parametrize("dtype", [L.FPO_BF16, L.FPO_F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name,m,address", [
    ("state1", 0, GRAD), ("state1", 0, GRAD + SIZE), ("W_master", 1, GRAD + SIZE), ("W_master", 1, GRAD),
    ("W_lp", 0, GRAD), ("W_lp", 1, GRAD + SIZE - 16), ("grad", 0, W - SIZE + 16), ("grad", 1, STATE + 2 * SIZE - 16),
    ("state1", 0, W), ("state1", 1, W), ("W_lp", 0, STATE), ("W_lp", 1, W), ("W_lp", 1, W + SIZE + 16),
    ("state1", 1, STATE + 64), ("W_master", 0, W + SIZE - 64)])
def test_muon_refuses_shared_buffers(lib, name, m, address, dtype):
    """The momentum pass overwrites what the conversion reads again; one batch's results
    are written before the next one's gradients are read."""
    status, message = muon(lib, dtype, **{name: (m, address)})
    assert status == L.FPO_ERR_ARG and "share memory" in message and name in message


def test_muon_without_a_state_in_use_is_refused_too(lib):
    assert muon(lib, momentum=0.0, state1=(0, GRAD))[0] == L.FPO_ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_muon_neighbours_and_repeated_gradients(dev, dtype):
    """Nothing between the buffers, a gradient given for two matrices, a float32 master that
    is its own copy: as with buffers of their own."""
    import torch

    from paper_2608_14563_amd import api
    lp = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, numel = 2, ROWS * COLS
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    arena = torch.randn(5 * numel, generator=g, device=dev)
    own = lambda k: arena[k * numel:(k + 1) * numel].view(ROWS, COLS)  # noqa: E731
    grad, W, state = [own(0)] * n, [own(1), own(2)], [own(3), own(4)]
    kept = arena.clone()
    alone = [[t.clone() for t in ts] for ts in (grad, W, state)]
    opt = api.MuonConfig(clip_frac=0.0, step=2)
    api.fpo_muon_update(opt, *alone, dtype=lp)
    api.fpo_muon_update(opt, grad, W, state, W_lp=W if dtype == "f32" else None, dtype=lp)
    assert torch.equal(own(0), kept[:numel].view(ROWS, COLS)) and not torch.equal(own(1), kept[numel:2 * numel].view(ROWS, COLS))
    for a, b in zip(alone, (grad, W, state)):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


# --------------------------------------------------------------------- layer norm
T, D = 16, 64
ROWS_X, ROW = T * D * 2, D * 2  # bytes of x or y, gain or bias in bf16


def layernorm(lib, T=T, **over):
    """Buffers that follow each other without a gap."""
    at = dict(x=BASE, gain=BASE + ROWS_X, bias=BASE + ROWS_X + ROW, y=BASE + ROWS_X + 2 * ROW)
    at["mean"] = at["y"] + ROWS_X
    at["rstd"] = at["mean"] + 4 * T
    at.update(over)
    desc = L.LnDesc(T, D, L.FPO_BF16, L.FPO_F32, 1e-5, 0.0)
    status = lib.fpo_layernorm(C.byref(desc), *[at[k] for k in ("x", "gain", "bias", "y", "mean", "rstd")], None)
    return status, lib.fpo_last_error().decode()


Y = BASE + ROWS_X + 2 * ROW


@pytest.mark.parametrize("name,address", [
    ("y", BASE + ROWS_X), ("y", BASE + ROWS_X + ROW), ("y", BASE + 16), ("y", BASE - ROWS_X + 16), ("mean", BASE),
    ("mean", BASE + ROWS_X - 4), ("mean", BASE + ROWS_X), ("rstd", BASE + ROWS_X + ROW), ("rstd", Y),
    ("rstd", Y + ROWS_X + 4), ("mean", Y + ROWS_X + 4 * T), ("gain", Y), ("bias", Y + ROWS_X - 16)])
def test_layernorm_refuses_shared_buffers(lib, name, address):
    status, message = layernorm(lib, **{name: address})
    assert status == L.FPO_ERR_ARG and "share memory" in message and name in message


def test_layernorm_of_one_row_refuses_its_gain_as_result(lib):
    assert layernorm(lib, T=1, y=BASE + ROWS_X)[0] == L.FPO_ERR_ARG


# --------------------------------------------------------------------- ranges that overlap in part
VX, VDY, VDX, VLP = BASE, BASE + ROWS_X, BASE + 3 * ROWS_X, BASE + 5 * ROWS_X
VG, VDG = BASE + 6 * ROWS_X, BASE + 6 * ROWS_X + ROW
VDB = VDG + 2 * ROW


def vjp(lib, **over):
    at = dict(x=VX, gain=VG, dy=VDY, dx=VDX, dx_lp=VLP, dgain=VDG, dbias=VDB)
    at.update(over)
    desc = L.LnDesc(T, D, L.FPO_BF16, L.FPO_F32, 1e-5, 0.0)
    status = lib.fpo_layernorm_vjp(C.byref(desc), *[at[k] for k in ("x", "gain", "dy", "dx", "dx_lp", "dgain", "dbias")], WS,
                                   1 << 30, None)
    return status, lib.fpo_last_error().decode()


@pytest.mark.parametrize("name,address", [
    ("dx", VX + 16), ("dx", VX - 2 * ROWS_X + 16), ("dx_lp", VDY + ROWS_X), ("dx_lp", VDX + ROWS_X), ("dgain", VG + 16),
    ("dgain", VDX + 256), ("dbias", VDG + 16), ("dbias", VLP + ROWS_X - 16), ("x", VDX + ROWS_X), ("dy", VLP - 16),
    ("gain", VDB + 16)])
def test_layernorm_vjp_refuses_partly_shared_buffers(lib, name, address):
    status, message = vjp(lib, **{name: address})
    assert status == L.FPO_ERR_ARG and "share memory" in message and name in message


@pytest.mark.parametrize("dtype", [L.FPO_BF16, L.FPO_F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,O", [((0, 1), (2, 2.5)), ((0, 1), (1.5, 3)), ((0, 1), (-0.5, 3)), ((0, 0), (0.5, 3))])
def test_orthogonalize_refuses_partly_shared_buffers(lib, M, O, dtype):
    """Places in units of one matrix; two sizes, of which each batch is written before the
    next one is read."""
    size = ROWS * COLS * (2 if dtype == L.FPO_BF16 else 4)
    at = lambda v: ptrs(*[BASE + int(k * size) for k in v])  # noqa: E731
    d = L.NsDesc(dtype, 5, 1e-7, None)
    status = lib.fpo_orthogonalize(C.byref(d), 2, i64(ROWS, ROWS // 2), i64(COLS, 2 * COLS), at(M), at(O), WS, 1 << 30, None)
    assert status == L.FPO_ERR_ARG and "share memory" in lib.fpo_last_error().decode()
