"""Refusals of fpo_orthogonalize, fpo_muon_update, fpo_layernorm and
fpo_layernorm_vjp, their workspace queries, and the rule that groups the
Newton-Schulz steps. Nothing here launches a kernel (CPU)."""
import ctypes as C
import math
import os
import shutil
import subprocess

import pytest

from paper_2608_14563_amd import _lib as L

FAKE = 0x100000  # aligned, never dereferenced: every call below fails validation first
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_14563_amd", "csrc")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.fail("libfpo.so is not built (run __graft_entry__.build())")
    return L.load()


def i64(*v):
    return (C.c_int64 * len(v))(*v)


def ptrs(*v):
    return (C.c_void_p * len(v))(*v)


def ns(dtype=L.FPO_BF16, steps=5, eps=1e-7, coef=None):
    return L.NsDesc(dtype, steps, eps, (C.c_double * len(coef))(*coef) if coef else None)


def orth(lib, desc, n=1, rows=(64,), cols=(128,), M=(FAKE,), O=(FAKE + 4096,), ws=FAKE, ws_bytes=1 << 40):
    return lib.fpo_orthogonalize(C.byref(desc) if desc else None, n, i64(*rows) if rows else None,
                                 i64(*cols) if cols else None, ptrs(*M) if M else None, ptrs(*O) if O else None, ws,
                                 ws_bytes, None)


def test_orthogonalize_refusals(lib):
    assert orth(lib, None) == L.FPO_ERR_NULL
    assert orth(lib, ns(), rows=None) == L.FPO_ERR_NULL
    assert orth(lib, ns(), M=None) == L.FPO_ERR_NULL
    assert orth(lib, ns(), O=(None,)) == L.FPO_ERR_NULL
    assert orth(lib, ns(dtype=2)) == L.FPO_ERR_DTYPE
    for n in (0, -1, 65):
        assert orth(lib, ns(), n=n) == L.FPO_ERR_SHAPE
    for r, c in ((0, 8), (8, 0), (-8, 8), (12, 8), (8, 20), (1, 8), (1 << 32, 8)):
        assert orth(lib, ns(), rows=(r,), cols=(c,)) == L.FPO_ERR_SHAPE
    assert orth(lib, ns(), rows=(1 << 15,), cols=((1 << 14) + 8,)) == L.FPO_ERR_UNSUPPORTED
    assert orth(lib, ns(), rows=(8,), cols=((1 << 23) + 8,)) == L.FPO_ERR_UNSUPPORTED  # 8 rows take 64
    assert orth(lib, ns(L.FPO_F32), rows=(1 << 14,), cols=((1 << 14) + 8,)) == L.FPO_ERR_UNSUPPORTED
    assert orth(lib, ns(L.FPO_F32), rows=(1 << 14,), cols=(1 << 14,), ws=None) == L.FPO_ERR_WORKSPACE
    for s in (0, -1, 33):
        assert orth(lib, ns(steps=s)) == L.FPO_ERR_ARG
    for e in (-1e-9, math.nan, math.inf):
        assert orth(lib, ns(eps=e)) == L.FPO_ERR_ARG
    assert orth(lib, ns(steps=1, coef=(1.0, math.nan, 0.0))) == L.FPO_ERR_ARG
    assert orth(lib, ns(steps=1, coef=(2000.0, 0.0, 0.0))) == L.FPO_ERR_ARG
    assert orth(lib, ns(steps=4, coef=(10.0, 0.0, 0.0) * 4)) == L.FPO_ERR_ARG  # 10, 100, 1000, 10^4
    assert "grow past" in lib.fpo_last_error().decode()
    assert orth(lib, ns(), M=(FAKE + 8,)) == L.FPO_ERR_ARG
    assert orth(lib, ns(), O=(FAKE + 2,)) == L.FPO_ERR_ARG
    assert orth(lib, ns(), ws=None) == L.FPO_ERR_WORKSPACE
    assert orth(lib, ns(), ws=FAKE + 16) == L.FPO_ERR_WORKSPACE
    need = lib.fpo_orthogonalize_workspace(C.byref(ns()), 1, i64(64), i64(128))
    assert need > 0 and orth(lib, ns(), ws_bytes=need - 1) == L.FPO_ERR_WORKSPACE


def test_a_buffer_given_twice_is_refused(lib):
    two = dict(n=2, rows=(64, 64), cols=(128, 128))
    assert orth(lib, ns(), M=(FAKE, FAKE), O=(FAKE + 64, FAKE + 64), **two) == L.FPO_ERR_ARG
    assert "same buffer" in lib.fpo_last_error().decode()
    C2 = FAKE + 128
    assert orth(lib, ns(), M=(C2, C2), O=(FAKE, FAKE + 64), ws=None, **two) == L.FPO_ERR_WORKSPACE  # M may repeat
    assert orth(lib, ns(), M=(C2, FAKE), O=(FAKE, FAKE + 64), **two) == L.FPO_ERR_ARG
    assert "is M of matrix 1" in lib.fpo_last_error().decode()
    A, B = FAKE, FAKE + 64
    for W, lp, st, want in (((A, A), (A, B), (A, B), L.FPO_ERR_ARG), ((A, B), (A, A), (A, B), L.FPO_ERR_ARG),
                            ((A, B), (A, B), (B, B), L.FPO_ERR_ARG), ((A, B), (A, B), (A, B), L.FPO_ERR_WORKSPACE)):
        u = L.UpdateBufs(ptrs(*W), ptrs(*lp), ptrs(*st), None, FAKE, None)
        assert lib.fpo_muon_update(C.byref(muon()), 2, i64(64, 64), i64(128, 128), ptrs(A, A), FAKE, C.byref(u), None, 0,
                                   None) == want


def test_orthogonalize_workspace(lib):
    def need(sizes, dtype=L.FPO_BF16, steps=5):
        d = ns(dtype, steps)
        return lib.fpo_orthogonalize_workspace(C.byref(d), len(sizes), i64(*[r for r, _ in sizes]),
                                               i64(*[c for _, c in sizes]))

    assert need([(64, 100)]) == 0  # refused
    one = need([(136, 328)])
    # two fp16 matrices n x m and five n x n, padded to 64
    assert one >= 2 * (2 * 192 * 384 + 5 * 192 * 192)
    assert need([(328, 136)]) == one and need([(136, 328)], steps=9) == one
    assert need([(136, 328)], L.FPO_F32) > one
    assert need([(136, 328), (64, 64)]) == max(one, need([(64, 64)]))  # batches take turns
    # a bounded number of large matrices at once
    assert need([(4096, 12288)] * 36) < 16 * need([(4096, 12288)])


def muon(**kw):
    f = dict(lr=1e-3, momentum=0.9, weight_decay=0.01, clip_frac=0.01, step=1, nesterov=1, scale=2, clip_target=0)
    nd = kw.pop("ns", ns())
    f.update(kw)
    return L.Muon(nd, *[f[k] for k in ("lr", "momentum", "weight_decay", "clip_frac", "step", "nesterov", "scale",
                                       "clip_target")])


def call_muon(lib, o, grad=(FAKE,), gsq=FAKE, W=(FAKE,), lp=(FAKE,), st=(FAKE,), wsq=FAKE, ws=FAKE, ws_bytes=1 << 40,
              rows=(64,), cols=(128,), upd=True):
    u = L.UpdateBufs(ptrs(*W) if W else None, ptrs(*lp) if lp else None, ptrs(*st) if st else None, None, wsq, None)
    return lib.fpo_muon_update(C.byref(o) if o else None, 1, i64(*rows), i64(*cols), ptrs(*grad) if grad else None, gsq,
                               C.byref(u) if upd else None, ws, ws_bytes, None)


def test_muon_refusals(lib):
    assert call_muon(lib, None) == L.FPO_ERR_NULL
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(momentum=1.5), dict(momentum=-0.1), dict(weight_decay=-1.0),
                dict(weight_decay=math.inf), dict(clip_frac=math.nan), dict(step=0), dict(nesterov=2), dict(scale=3),
                dict(scale=-1), dict(clip_target=2), dict(ns=ns(steps=0)), dict(ns=ns(eps=-1.0))):
        assert call_muon(lib, muon(**bad)) == L.FPO_ERR_ARG, bad
    assert call_muon(lib, muon(ns=ns(dtype=5))) == L.FPO_ERR_DTYPE
    assert call_muon(lib, muon(), rows=(60,)) == L.FPO_ERR_SHAPE
    for over in (dict(grad=None), dict(W=None), dict(upd=False), dict(grad=(None,)), dict(W=(None,)), dict(st=None),
                 dict(st=(None,)), dict(wsq=None), dict(gsq=None)):
        assert call_muon(lib, muon(), **over) == L.FPO_ERR_NULL, over
    for over in (dict(grad=(FAKE + 4,)), dict(W=(FAKE + 8,)), dict(st=(FAKE + 4,)), dict(lp=(FAKE + 4,))):
        assert call_muon(lib, muon(), **over) == L.FPO_ERR_ARG, over
    assert call_muon(lib, muon(), lp=(FAKE + 8,), ws=None) == L.FPO_ERR_WORKSPACE  # 8 bytes are enough for bf16
    assert call_muon(lib, muon(ns=ns(L.FPO_F32)), lp=(FAKE + 8,)) == L.FPO_ERR_ARG
    # what may be left out: the next complaint is the workspace
    for o, over in ((muon(momentum=0.0), dict(st=None)), (muon(momentum=0.0), dict(st=(None,))),
                    (muon(clip_frac=0.0), dict(wsq=None, gsq=None)), (muon(clip_target=1), dict(gsq=None)),
                    (muon(), dict(lp=None)), (muon(), dict(lp=(None,)))):
        assert call_muon(lib, o, ws=None, **over) == L.FPO_ERR_WORKSPACE
    assert lib.fpo_muon_update_workspace(C.byref(muon()), 1, i64(64), i64(128)) == lib.fpo_orthogonalize_workspace(
        C.byref(ns()), 1, i64(64), i64(128))
    assert lib.fpo_muon_update_workspace(C.byref(muon(lr=-1.0)), 1, i64(64), i64(128)) == 0


def ln(T=4, d=64, dtype=L.FPO_BF16, dy=L.FPO_F32, eps=1e-5, min_std=0.0):
    return L.LnDesc(T, d, dtype, dy, eps, min_std)


def test_layernorm_refusals(lib):
    def fwd(desc, x=FAKE, gain=FAKE, bias=FAKE, y=FAKE + 256):
        return lib.fpo_layernorm(C.byref(desc) if desc else None, x, gain, bias, y, None, None, None)

    def vjp(desc, x=FAKE, gain=FAKE, dy=FAKE, dx=FAKE + 256, lp=FAKE + 512, dg=FAKE + 768, db=FAKE + 1024, ws=FAKE,
            ws_bytes=1 << 40):
        return lib.fpo_layernorm_vjp(C.byref(desc) if desc else None, x, gain, dy, dx, lp, dg, db, ws, ws_bytes, None)

    for f in (fwd, vjp):
        assert f(None) == L.FPO_ERR_NULL
        assert f(ln(), x=None) == L.FPO_ERR_NULL
        for bad in (dict(T=0), dict(T=-1), dict(d=0), dict(d=60), dict(T=(1 << 23) + 1), dict(d=(1 << 22) + 8)):
            assert f(ln(**bad)) == L.FPO_ERR_SHAPE, bad
        for bad in (dict(eps=-1.0), dict(eps=math.nan), dict(min_std=-1.0), dict(min_std=math.inf)):
            assert f(ln(**bad)) == L.FPO_ERR_ARG, bad
        for bad in (dict(dtype=2), dict(dy=-1)):
            assert f(ln(**bad)) == L.FPO_ERR_DTYPE, bad
        assert f(ln(), x=FAKE + 8) == L.FPO_ERR_ARG
        assert f(ln(), gain=FAKE + 2) == L.FPO_ERR_ARG
    assert fwd(ln(), y=None) == L.FPO_ERR_NULL and fwd(ln(), y=FAKE + 4) == L.FPO_ERR_ARG
    assert fwd(ln(), bias=FAKE + 4) == L.FPO_ERR_ARG
    assert vjp(ln(), dy=None) == L.FPO_ERR_NULL and vjp(ln(), dy=FAKE + 4) == L.FPO_ERR_ARG
    assert vjp(ln(), dx=None, lp=None, dg=None, db=None) == L.FPO_ERR_NULL
    for k in ("dx", "lp", "dg", "db"):
        assert vjp(ln(), **{k: FAKE + 4}) == L.FPO_ERR_ARG
    assert fwd(ln(), y=FAKE) == L.FPO_ERR_ARG
    for k in ("dx", "lp", "dg", "db"):
        assert vjp(ln(T=600), **{k: FAKE}) == L.FPO_ERR_ARG
        assert "one of the inputs" in lib.fpo_last_error().decode()
    assert vjp(ln(T=600), lp=FAKE + 256) == L.FPO_ERR_ARG and vjp(ln(T=600), db=FAKE + 768) == L.FPO_ERR_ARG
    assert vjp(ln(T=600), ws=None) == L.FPO_ERR_WORKSPACE
    assert vjp(ln(T=600), ws_bytes=16) == L.FPO_ERR_WORKSPACE
    assert vjp(ln(T=600), ws=FAKE + 4) == L.FPO_ERR_WORKSPACE


def test_layernorm_workspace(lib):
    def need(T, d):
        return lib.fpo_layernorm_vjp_workspace(C.byref(ln(T, d)))

    assert need(0, 64) == 0 and need(1, 64) == 0 and need(4, 64) == 0  # one workgroup's sums are the results
    assert need(17, 512) >= 5 * 2 * 512 * 4  # a wave a row, four to a workgroup
    assert need(1 << 23, 4096) == need(1 << 20, 4096) <= 64 << 20


# --------------------------------------------------------------------- the binding's own checks
def test_binding_refusals():
    import torch

    from paper_2608_14563_amd import api
    a = torch.zeros(8, 8)
    with pytest.raises(ValueError):
        api.fpo_orthogonalize([], [])
    with pytest.raises(ValueError):
        api.fpo_orthogonalize([a], [a], coefs=[(1.0, 0.0, 0.0)] * 3)
    with pytest.raises(ValueError):
        api.fpo_orthogonalize([a], [a], coefs=[(1.0, 0.0)] * 5)
    with pytest.raises(ValueError):
        api.fpo_orthogonalize_workspace([(8,)], torch.float32)
    with pytest.raises(TypeError):
        api.fpo_orthogonalize([a.double()], [a.double()])
    with pytest.raises(ValueError):
        api.fpo_muon_update(api.MuonConfig(), [], [], [])
    with pytest.raises(TypeError):
        api.fpo_layernorm(a.half(), None, None, a.half())
    for call in (lambda: api.fpo_layernorm(a, None, None, a), lambda: api.fpo_orthogonalize([a], [a]),
                 lambda: api.fpo_muon_update(api.MuonConfig(), [a], [a], [a]),
                 lambda: api.fpo_layernorm_vjp(a, None, a, dx=a)):
        with pytest.raises(ValueError):  # CPU tensors
            call()


# --------------------------------------------------------------------- groups and exponents
SRC = """
#include "ns.hpp"
extern "C" int plan(int steps, const double* coef, int first, int* out) {  // per group: count, e_X; per step: e_A, e_B, e_C, e_Q
  const fpo::NsPlan p = fpo::ns_plan(steps, coef, first);
  if (!p.ok) return -1;
  for (int i = 0; i < p.ngroups; ++i) { *out++ = p.groups[i].first; *out++ = p.groups[i].count; *out++ = p.groups[i].e_X; }
  for (int i = 0; i < p.nsteps; ++i) { const fpo::NsStep& s = p.steps[i]; *out++ = s.e_A; *out++ = s.e_B; *out++ = s.e_C; *out++ = s.e_Q; }
  *out = p.e_out;
  return p.ngroups;
}
extern "C" double value_max(double a, double b, double c, double top) { return fpo::ns_value_max(a, b, c, top); }
extern "C" double poly_max(double a, double b, double c, double top) { return fpo::ns_poly_max(a, b, c, top); }
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("ns")
    (d / "ns.cpp").write_text(SRC)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-shared", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__=1", "-I",
                    os.path.join(rocm, "include"), "-I", CSRC, str(d / "ns.cpp"), "-o", str(d / "ns.so")], check=True)
    lib = C.CDLL(str(d / "ns.so"))
    lib.value_max.restype = lib.poly_max.restype = C.c_double
    lib.value_max.argtypes = lib.poly_max.argtypes = [C.c_double] * 4
    return lib


def plan(host, steps, coef=None, first=2):
    out = (C.c_int * 512)()
    n = host.plan(steps, (C.c_double * (3 * steps))(*coef) if coef else None, first, out)
    if n < 0:
        return None
    g = [tuple(out[3 * i:3 * i + 3]) for i in range(n)]
    s = [tuple(out[3 * n + 4 * i:3 * n + 4 * i + 4]) for i in range(steps)]
    return g, s, out[3 * n + 4 * steps]


def test_groups(host):
    counts = lambda k, first, c=None: [g[1] for g in plan(host, k, c, first)[0]]  # noqa: E731
    for first in (1, 2, 3):
        assert counts(1, first) == [1] and counts(2, first) == [min(first, 2)] + [1] * (first == 1)
        # coefficients that enlarge more: groups close earlier
        assert counts(3, first, (13.0, -40.0, 28.0) + (1.5, -0.5, 0.0) * 2)[0] == 1
        for k in range(1, 33):
            g = plan(host, k, None, first)[0]
            assert sum(c for _, c, _ in g) == k
            assert [f for f, _, _ in g] == [sum(c for _, c, _ in g[:i]) for i in range(len(g))]
    assert counts(5, 1) == [1] * 5
    assert counts(3, 2) == [2, 1] and counts(5, 2) == [2, 1, 2] and counts(7, 2) == [2, 1, 2, 1, 1]
    assert counts(3, 3) == [3] and counts(5, 3) == [3, 2] and counts(7, 3) == [3, 2, 1, 1]
    assert plan(host, 2, (100.0, 0.0, 0.0) * 2) is None


def test_bounds_and_exponents(host):
    """The bounds hold at every point, and every stored matrix stays under 2^13 of fp16's 65504."""
    import numpy as np
    rng = np.random.default_rng(0)
    coefs = [(3.4445, -4.775, 2.0315), (1.5, -0.5, 0.0), (1.0, 0.0, 0.0), (-2.0, 3.0, -1.0), (0.0, 0.0, 0.5),
             (8.0, -23.0, 17.0)] + [tuple(rng.normal(size=3) * 3) for _ in range(50)]
    for a, b, c in coefs:
        for top in (0.3, 1.0, 1.3, 4.0):
            s = np.linspace(0, top, 20001)
            v, w = np.abs(a * s + b * s ** 3 + c * s ** 5).max(), np.abs(a + b * s ** 2 + c * s ** 4).max()
            assert v <= host.value_max(a, b, c, top) * (1 + 1e-12) <= v * (1 + 1e-6) + 1e-12
            assert w <= host.poly_max(a, b, c, top * top) * (1 + 1e-12) <= w * (1 + 1e-6) + 1e-12
    for k, coef in ((5, None), (7, None), (3, (13.0, -40.0, 28.0) + (1.5, -0.5, 0.0) * 2), (12, (1.5, -0.5, 0.0) * 12)):
        groups, steps, e_out = plan(host, k, coef, 3 if k % 2 else 2)
        lam = np.linspace(0, 1, 4001)  # eigenvalues of A
        for first, count, e_x in groups:
            assert np.sqrt(lam).max() * 2.0 ** e_x <= 2 ** 13
            q = np.ones_like(lam)
            for j in range(first, first + count):
                a, b, c = (coef or (3.4445, -4.775, 2.0315) * k)[3 * j:3 * j + 3]
                e_a, e_b, e_c, e_q = steps[j]
                B = a + b * lam + c * lam ** 2
                q = q * B
                for v, e in ((lam, e_a), (B, e_b), (B * lam, e_c), (q, e_q)):
                    assert np.abs(v).max() * 2.0 ** e <= 2 ** 13
                lam = lam * B * B
        assert np.sqrt(lam).max() * 2.0 ** e_out <= 2 ** 13


def test_call_makes_the_tensors_device_current(monkeypatch):
    import torch

    from paper_2608_14563_amd import api
    seen = []

    class Device:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            seen.append(("enter", self.d))

        def __exit__(self, *a):
            seen.append("exit")

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(api, "_current_device", lambda: 0)
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    api._call(here, lambda x: seen.append(x) or 0, 5)
    assert seen == [5]
    api._call(there, lambda x: seen.append(x) or 0, 6)
    assert seen == [5, ("enter", there), 6, "exit"]
    with pytest.raises(L.FpoError):
        api._call(here, lambda: L.FPO_ERR_ARG)
