"""Orthogonal updates without a GPU: refusals, sizes, and the reference the GPU tests compare with."""
import ctypes as C
import os

import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import orth_ref as ref

GOOD, OTHER, ODD = 0x10000, 0x20000, 0x10004


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(nf.LIB_PATH):
        from paper_2402_14139_amd import build
        build.build()
    return nf.lib()


def _arr(*p):
    return (C.c_void_p * len(p))(*p)


def _dims(*v):
    return (C.c_int32 * len(v))(*v)


def _with(**kw):
    d = nf.orth_desc(ref.MUON)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("desc,n,rows,cols,status", [
    (dict(steps=0), 1, 8, 8, nf.NF_ERR_BAD_DESC), (dict(steps=13), 1, 8, 8, nf.NF_ERR_BAD_DESC), (dict(steps=-1), 1, 8, 8, nf.NF_ERR_BAD_DESC),
    (dict(eps=-1e-9), 1, 8, 8, nf.NF_ERR_BAD_DESC), (dict(eps=float("nan")), 1, 8, 8, nf.NF_ERR_BAD_DESC),
    (dict(), 0, 8, 8, nf.NF_ERR_BAD_DESC), (dict(), 33, 8, 8, nf.NF_ERR_BAD_DESC), (dict(), 1, 0, 8, nf.NF_ERR_BAD_DESC), (dict(), 1, 8, -1, nf.NF_ERR_BAD_DESC),
    (dict(), 1, (1 << 20) + 1, 8, nf.NF_ERR_UNSUPPORTED), (dict(), 1, 8, (1 << 20) + 1, nf.NF_ERR_UNSUPPORTED),
    (dict(), 1, (1 << 14) + 1, (1 << 14) + 1, nf.NF_ERR_UNSUPPORTED)])
def test_descriptors(L, desc, n, rows, cols, status):
    d, out = _with(**desc), C.c_size_t()
    r, c = _dims(*[rows] * 33), _dims(*[cols] * 33)
    p, q = _arr(*[GOOD + 256 * i for i in range(33)]), _arr(*[OTHER + 256 * i for i in range(33)])
    assert L.nf_orthogonalise_workspace_bytes(C.byref(d), n, r, c, C.byref(out)) == status
    assert L.nf_orthogonalise(C.byref(d), 0, n, p, q, r, c, GOOD, 1 << 60, None) == status
    m = nf.MuonDesc(lr=0.1, momentum=0.9, orth=d)
    assert L.nf_muon_update(C.byref(m), n, p, q, p, r, c, GOOD, 1 << 60, None) == status


@pytest.mark.parametrize("steps,good", [
    (ref.MUON, True), (ref.CUBIC, True), (ref.QUINTIC, True), ([(8.3, -23.6, 17.3), (4.1, -2.9, 0.5)], True), ([(0.0, 0.0, 0.0)] * 3, True), ([(1.0, 0.0, 0.0)] * 12, True),
    ([(100.0, 0.0, 0.0)] * 5, False), ([(1.0, 1.0, 1.0)] * 12, False), ([(float("nan"), 0.0, 0.0)], False), ([(float("inf"), 0.0, 0.0)], False),
    ([(1.0, float("nan"), 0.0)], False), ([(1.0, 0.0, float("-inf"))], False)])
def test_unbounded_steps_are_refused(L, steps, good):
    d, out = nf.orth_desc(steps), C.c_size_t()
    assert L.nf_orthogonalise_workspace_bytes(C.byref(d), 1, _dims(8), _dims(8), C.byref(out)) == (nf.NF_OK if good else nf.NF_ERR_UNSUPPORTED)


def test_pointers(L):
    d = _with()
    need = nf.nf_orthogonalise_workspace_bytes(d, [(16, 27), (64, 64)])
    r, c = _dims(16, 64), _dims(27, 64)
    two = _arr(GOOD, OTHER)
    swapped, apart = _arr(OTHER, GOOD), _arr(GOOD + 0x100000, OTHER + 0x100000)
    def orth(g=two, y=apart, rows=r, cols=c, ws=GOOD, n=need, dt=0, desc=C.byref(d)):
        return L.nf_orthogonalise(desc, dt, 2, g, y, rows, cols, ws, n, None)
    for k in ("g", "y", "rows", "cols", "desc"):
        assert orth(**{k: None}) == nf.NF_ERR_NULL
    assert orth(g=_arr(GOOD, None)) == orth(y=_arr(None, GOOD)) == nf.NF_ERR_NULL
    assert orth(g=_arr(GOOD, ODD)) == orth(y=_arr(ODD, GOOD)) == orth(y=_arr(0x900000, 0x900000)) == orth(y=swapped) == orth(dt=3) == orth(dt=-1) == nf.NF_ERR_BAD_DESC
    assert orth(ws=None) == orth(ws=0x10010) == orth(n=need - 1) == nf.NF_ERR_WORKSPACE
    m = nf.MuonDesc(lr=0.1, momentum=0.9, weight_decay=0.0, nesterov=1, orth=d)
    others, third = _arr(GOOD + 0x200000, OTHER + 0x200000), _arr(GOOD + 0x300000, OTHER + 0x300000)
    def muon(w=two, g=others, v=third, rows=r, cols=c, ws=GOOD, n=need, desc=C.byref(m)):
        return L.nf_muon_update(desc, 2, w, g, v, rows, cols, ws, n, None)
    for k in ("w", "g", "rows", "cols", "desc"):
        assert muon(**{k: None}) == nf.NF_ERR_NULL
    assert muon(w=_arr(GOOD, GOOD)) == muon(v=_arr(GOOD, GOOD)) == muon(v=_arr(GOOD, ODD)) == muon(w=_arr(ODD, GOOD)) == muon(g=_arr(ODD, GOOD)) == nf.NF_ERR_BAD_DESC
    for k in (dict(g=two), dict(v=two), dict(v=_arr(GOOD + 0x300000, GOOD)), dict(g=_arr(GOOD + 0x100000, GOOD)), dict(v=others), dict(v=_arr(OTHER + 0x200000, GOOD + 0x300000))):
        assert muon(**k) == nf.NF_ERR_BAD_DESC   # what is written is nothing else's
    assert muon(v=_arr(GOOD, None)) == nf.NF_ERR_NULL
    assert muon(ws=None) == muon(n=need - 1) == nf.NF_ERR_WORKSPACE
    assert nf.nf_orthogonalise_workspace_bytes(d, [(16, 27)]) <= need
    assert L.nf_orthogonalise_workspace_bytes(C.byref(d), 2, r, c, None) == nf.NF_ERR_NULL


@pytest.mark.parametrize("rows,cols", [(5, 9), (9, 5), (7, 7), (1, 4), (4, 1)])
def test_reference_against_singular_values(rows, cols):
    g = torch.randn(rows, cols, generator=torch.Generator().manual_seed(rows), dtype=torch.float64)
    f32 = lambda steps: [tuple(float(torch.tensor(v, dtype=torch.float32)) for v in s) for s in steps]  # noqa: E731
    for steps in (ref.MUON, ref.CUBIC, ref.QUINTIC):
        assert torch.allclose(ref.steps(g, steps, 1e-7), ref.by_singular_values(g, f32(steps), 1e-7), atol=1e-9)
    y = ref.steps(g, ref.CUBIC, 0.0)
    assert torch.allclose(y @ y.t() if rows <= cols else y.t() @ y, torch.eye(min(rows, cols), dtype=torch.float64), atol=1e-2)
