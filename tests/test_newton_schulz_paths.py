"""The Newton-Schulz kernels that each batch size runs, on dense matrices against float64:
which path a case takes is asserted on the host (CPU), so that a changed estimate cannot
move a case off the kernels it is here for, and its results on the GPU.

Tolerances (Frobenius norms). FPO_BF16: twice what the iteration loses in the groups that
the case runs in when every matrix it stores (X, A, B, B A, the products of the B) is
rounded once to fp16, evaluated on the same input. The kernels store the same matrices
and keep besides what the diagonals lose, which only helps; twice, because their float32
sums round too and because a rounding that falls differently is enlarged like the first
one. A bf16 result adds its own rounding: that of the float64 result, 5% more because it
is another sample of the same distribution (over a million entries differ by less).
FPO_F32: a sum of K products rounds its accumulator 3 K times (three products), at
random sqrt(3 K) 2^-24 altogether; sixteen times that for the five steps and what a
group's B A B enlarges, on matrices whose singular values keep away from zero."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import operators as P
from paper_2608_14563_amd import _lib as L
from paper_2608_14563_amd import api
from tests._util import host64

BF, F32 = torch.bfloat16, torch.float32
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_14563_amd", "csrc")

# rows, cols (half of them the other way round with `turned`), matrices, type: steps in each
# group; tiles of X X^T, an n x n product, two of them in a launch, the product with X (with
# small tiles the waves a tile; + 128: the last ones as quarters; r: tiles past the edges)
CASES = {
    "128 tiles": (1000, 2744, 4, BF, False, (3, 2), ("128", "128", "128", "256r")),
    "whole tiles and quarters": (2048, 3200, 8, BF, False, (3, 2), ("256+128", "256+128", "256+128", "256r+128")),
    "both ways": (2048, 4096, 8, BF, True, (3, 2), ("256+128", "256+128", "256+128", "256")),
    "ragged": (1288, 2056, 7, BF, True, (3, 2), ("128", "128", "256r+128", "256r+128")),
    "ragged in float32": (1000, 2744, 4, F32, True, (2, 1, 2), ("128", "128", "128", "256r")),
    "whole tiles in float32": (2048, 3200, 8, F32, False, (2, 1, 2), ("256+128", "256+128", "256+128", "256r+128")),
    "small, two a group": (384, 1032, 9, BF, True, (2, 1, 2), ("8", "8", "", "4")),
    "small, four waves": (296, 600, 20, BF, True, (2, 1, 2), ("4", "4", "", "4")),
    "small, four waves, wide": (512, 1376, 8, BF, False, (2, 1, 2), ("4", "4", "", "4")),
    "small, four waves, one a group": (320, 328, 20, BF, False, (1, 1, 1, 1, 1), ("4", "4", "", "4")),
    "small, float32": (296, 600, 20, F32, True, (2, 1, 2), ("4", "4", "", "4")),
    "small, float32, one a group": (320, 328, 20, F32, False, (1, 1, 1, 1, 1), ("4", "4", "", "4")),
}

SRC = """
#include "ns.hpp"
using namespace fpo;
extern "C" int choose(long n, long m, int count, int bf16, int steps, const double* coef, int* groups) {
  const NsChoice c = ns_choose(n, m, count, bf16 != 0);  // (groups: steps of each, then 0)
  const NsPlan p = ns_plan(steps, coef, c.first);
  for (int i = 0; i < p.ngroups; ++i) groups[i] = p.groups[i].count;
  groups[p.ngroups] = 0;
  return c.small;
}
extern "C" long big_tiles(long M, long N, long K, long mats, int sym, long* all) {
  const NsSplit s = ns_split(M, N, K, mats, sym != 0);
  *all = mats * ns_tiles(M, N, s.nbig ? 256 : 128, sym != 0);
  return s.nbig;
}
extern "C" long small_tiles(long M, long N, int sym) { return ns_tiles(M, N, 64, sym != 0); }
extern "C" int batch_limit(long n) { return ns_batch_limit(n); }
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("ns_paths")
    (d / "ns.cpp").write_text(SRC)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-shared", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__=1", "-I",
                    os.path.join(rocm, "include"), "-I", CSRC, str(d / "ns.cpp"), "-o", str(d / "ns.so")], check=True)
    lib = C.CDLL(str(d / "ns.so"))
    lib.big_tiles.restype = lib.small_tiles.restype = C.c_long
    lib.big_tiles.argtypes = [C.c_long] * 4 + [C.c_int, C.POINTER(C.c_long)]
    lib.small_tiles.argtypes = [C.c_long, C.c_long, C.c_int]
    lib.choose.argtypes = [C.c_long, C.c_long, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int)]
    lib.batch_limit.argtypes = [C.c_long]
    return lib


def groups_of(host, short, longer, n, bf16, per_step=(P.MUON_COEF,) * 5):
    """(small tiles, steps in each group)"""
    g = (C.c_int * 64)()
    flat = [v for k in per_step for v in k]
    small = host.choose(short, longer, n, bf16, len(per_step), (C.c_double * len(flat))(*flat), g)
    return small, tuple(g[:list(g).index(0)])


def path(host, rows, cols, n, dtype):
    """(steps of the groups, tiles of the launches) of n matrices, as CASES states them."""
    short, longer, bf16 = min(rows, cols), max(rows, cols), dtype == BF
    assert n <= host.batch_limit(short)  # one batch
    small, groups = groups_of(host, short, longer, n, bf16)
    np_, mp = (-(-v // 64) * 64 for v in (short, longer))
    launches = ((np_, np_, mp, 1, 1), (np_, np_, np_, 1, 1), (np_, np_, np_, 2, 1), (np_, mp, np_, 1, 0))
    out = []
    for M, N, K, sets, sym in launches:
        if small:
            out.append("" if sets == 2 else "8" if n * host.small_tiles(M, N, sym) <= 256 else "4")
            continue
        every = C.c_long()
        big = host.big_tiles(M, N, K * (1 if bf16 else 3), n * sets, sym, C.byref(every))
        out.append("128" if not big else "256" + "r" * bool(M % 256 or N % 256) + "+128" * (big < every.value))
    return groups, tuple(out)


@pytest.mark.parametrize("name", CASES)
def test_paths(host, name):
    rows, cols, n, dtype, _, groups, launches = CASES[name]
    assert path(host, rows, cols, n, dtype) == (groups, launches)


def test_small_tiles_take_one_set_of_operands(host):
    """Their groups have two steps at most: no launch multiplies two sets of operands."""
    for n in range(8, 1025, 56):
        for m in range(n, 4 * n + 1, 56):
            for count in (1, 2, 5, 9, 20, 64):
                for bf16 in (0, 1):
                    small, groups = groups_of(host, n, m, count, bf16)
                    if small:
                        assert max(groups) <= 2


# --------------------------------------------------------------------- float64 on the GPU
def to_fp16(x):
    return (x * 512).half().double() / 512


def iterate(M, groups, store=lambda x: x, per_step=(P.MUON_COEF,) * 5):
    """The steps in float64, in the given groups, `store` applied to every matrix kept."""
    X = M.double()
    X = X if X.shape[0] <= X.shape[1] else X.t().contiguous()
    X = X / (X.square().sum().sqrt() + 1e-7)
    eye, at = torch.eye(X.shape[0], dtype=torch.float64, device=X.device), 0
    for count in groups:
        X = store(X)
        A, Q = store(X @ X.t()), None
        for j in range(count):
            a, b, c = per_step[at]
            at += 1
            B = store(a * eye + b * A + c * (A @ A))
            Q = B if Q is None else store(B @ Q)
            if j + 1 < count:
                A = store(store(B @ A) @ B)
        X = Q @ X
    return X if M.shape[0] <= M.shape[1] else X.t()


def reference(M, groups, dtype, per_step=(P.MUON_COEF,) * 5):
    """(float64 result, tolerance of the unrounded direction)."""
    E = iterate(M, (1,) * len(per_step), per_step=per_step)
    if dtype == F32:
        return E, 16 * (3 * max(M.shape)) ** 0.5 * 2 ** -24 * E.norm().item()
    return E, 2 * (iterate(M, groups, to_fp16, per_step) - E).norm().item()


def matrix(shape, kind, g, dev):
    r, c = shape
    rand = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    n = min(r, c)
    if kind == "normal":
        return rand(r, c)
    if kind == "rank":  # a quarter of the directions
        return rand(r, n // 4) @ rand(n // 4, c)
    if kind == "tokens":  # a sum over tokens of unequal weight
        return (rand(r, 2 * n) * torch.exp(0.5 * rand(1, 2 * n))) @ rand(2 * n, c)
    assert kind == "decay"  # singular values 1 / k
    U, V = (torch.linalg.qr(rand(s, n).double())[0] for s in (r, c))
    return ((U / torch.arange(1, n + 1, device=dev)) @ V.t()).float()


def shapes_of(rows, cols, n, turned):
    return [(cols, rows) if turned and i % 2 else (rows, cols) for i in range(n)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_orthogonalize(dev, name):
    rows, cols, n, dtype, turned, groups, _ = CASES[name]
    g = torch.Generator(device=dev)
    g.manual_seed(rows + cols)
    kinds = ("normal", "decay", "rank", "tokens") if dtype == BF else ("normal",)
    M = [matrix(s, kinds[i % len(kinds)], g, dev).to(dtype) for i, s in enumerate(shapes_of(rows, cols, n, turned))]
    O = [torch.full_like(m, float("nan")) for m in M]
    api.fpo_orthogonalize(M, O)
    for i in sorted({0, 1, 2, 3, n // 2, n - 1}):
        E, tol = reference(M[i], groups, dtype)
        own = 1.05 * (E.to(dtype).double() - E).norm().item()
        off = (O[i].double() - E).norm().item()
        assert off <= tol + own, f"{kinds[i % len(kinds)]} matrix {i}: off by {off:.3e}, allowed {tol:.3e} + {own:.3e}"



# case, coefficients of each step: steps in each group
D, CUBIC, VARIED = P.MUON_COEF, (1.5, -0.5, 0.0), ((4.0, -7.0, 4.0), P.MUON_COEF, (1.875, -1.25, 0.375))
STEPS = [("128 tiles", (D,), (1,)), ("128 tiles", (D,) * 3, (3,)), ("128 tiles", (D,) * 4, (3, 1)),
         ("128 tiles", (D,) * 6, (3, 2, 1)), ("128 tiles", (CUBIC,) * 12, (3, 2, 1, 2, 1, 2, 1)), ("128 tiles", VARIED, (2, 1)),
         ("small, two a group", (D,) * 2, (2,)), ("small, two a group", (D,) * 4, (2, 1, 1)),
         ("small, two a group", (D,) * 6, (2, 1, 2, 1)), ("small, two a group", VARIED, (2, 1))]


@pytest.mark.parametrize("name,per_step,groups", STEPS)
def test_groups(host, name, per_step, groups):
    rows, cols, n = CASES[name][:3]
    assert groups_of(host, min(rows, cols), max(rows, cols), n, 1, per_step)[1] == groups


@pytest.mark.gpu
@pytest.mark.parametrize("name,per_step,groups", STEPS)
def test_steps_and_coefficients(dev, name, per_step, groups):
    rows, cols, n, dtype, turned = CASES[name][:5]
    g = torch.Generator(device=dev)
    g.manual_seed(rows + len(per_step))
    M = [matrix(s, "normal", g, dev).to(dtype) for s in shapes_of(rows, cols, n, turned)]
    O = [torch.full_like(m, float("nan")) for m in M]
    api.fpo_orthogonalize(M, O, steps=len(per_step), coefs=per_step)
    for i in (0, n - 1):
        E, tol = reference(M[i], groups, dtype, per_step)
        own = 1.05 * (E.to(dtype).double() - E).norm().item()
        off = (O[i].double() - E).norm().item()
        assert off <= tol + own, f"matrix {i}: off by {off:.3e}, allowed {tol:.3e} + {own:.3e}"


CLIPS = {"off": dict(clip_frac=0.0), "gradient": dict(clip_frac=0.01, clip_target=L.FPO_CLIP_GRADIENT),
         "update": dict(clip_frac=0.01, clip_target=L.FPO_CLIP_UPDATE)}


@pytest.mark.gpu
@pytest.mark.parametrize("clip", CLIPS)
@pytest.mark.parametrize("name", ["whole tiles and quarters", "both ways", "ragged", "ragged in float32", "small, four waves"])
def test_muon(dev, name, clip):
    """The step against float64: the direction counts, at this learning rate a fifth of W."""
    rows, cols, n, dtype, turned, groups, _ = CASES[name]
    shapes = shapes_of(rows, cols, n, turned)
    g = torch.Generator(device=dev)
    g.manual_seed(rows + cols + 1)
    opt = api.MuonConfig(lr=2e-2, step=3, **CLIPS[clip])
    rand = lambda s, k: k * torch.randn(*s, generator=g, device=dev)  # noqa: E731
    kinds = ("normal", "tokens") if dtype == BF else ("normal",)
    grad = [matrix(s, kinds[i % len(kinds)], g, dev) for i, s in enumerate(shapes)]
    grad = [x * (1e-2 / x.std()) for x in grad]
    W = [rand(s, 0.02) for s in shapes]
    buf = [rand(s, 3e-4 if clip == "gradient" else 1e-2) for s in shapes]  # (the clip makes the gradient 2e-4)
    sumsq = lambda ts: torch.stack([t.double().square().sum() for t in ts])  # noqa: E731
    W_sumsq, grad_sumsq = sumsq(W), sumsq(grad)
    W_lp = [torch.full(s, float("nan"), dtype=dtype, device=dev) for s in shapes]
    factor = torch.full((n,), float("nan"), device=dev)
    W0, b0, g0 = ([t.clone() for t in ts] for ts in (W, buf, grad))
    api.fpo_muon_update(opt, grad, W, buf, W_sumsq=W_sumsq, grad_sumsq=grad_sumsq if clip == "gradient" else None,
                        W_lp=W_lp, clip_scale=factor, dtype=dtype)
    for i in sorted({0, 1, n // 2, n - 1}):
        w, d, b = host64(W0[i]), host64(g0[i]), host64(b0[i])
        args = (w, d, b, opt.lr, opt.momentum, True, opt.weight_decay, "rms", opt.step, opt.clip_frac,
                "update" if clip == "update" else "gradient")
        u = P.muon(*args, orthogonal=np.zeros_like(w))[3]
        E, tol = reference(torch.from_numpy(u).to(dev), groups, dtype)
        want, b1, k, _ = P.muon(*args, orthogonal=E.cpu().numpy())
        size = opt.lr * P.muon_scale("rms", *w.shape)
        # the direction's error, and float32 roundings of decay, product and sum. The update clip's factor k scales
        # the step, and with it its error, and is itself off by the step's; the gradient clip's k scales u, whose
        # direction O has the same size at any k
        slack = size * tol * (2 * k if clip == "update" else 1) + 4 * 2 ** -24 * (np.linalg.norm(w) + size * E.norm().item())
        off = np.linalg.norm(host64(W[i]) - want)
        assert off <= slack, f"matrix {i}: W off by {off:.3e}, allowed {slack:.3e}"
        assert off <= 0.05 * np.linalg.norm(want - w)  # (what is compared is the step, not W)
        g_scale = k if clip == "gradient" else 1.0  # (only this clip scales what enters the momentum)
        bound = 3 * 2 ** -24 * (opt.momentum * np.abs(b) + g_scale * np.abs(d)) + 1e-30
        assert bool((np.abs(host64(buf[i]) - b1) <= bound).all()), f"matrix {i}: momentum"
        rel = 1e-6 + (tol / E.norm().item() if clip == "update" else 0)
        assert abs(float(factor[i]) - k) <= rel * k and (k < 1) == (clip != "off")
        w1 = host64(W[i])
        assert abs(float(W_sumsq[i]) - (w1 * w1).sum()) <= 1e-12 * (w1 * w1).sum()
    for i in range(n):
        assert torch.equal(grad[i], g0[i]) and torch.equal(W_lp[i], W[i].to(dtype))
