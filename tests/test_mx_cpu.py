"""Matrices in 4 bits without a GPU: refusals, sizes, and the reference the GPU tests compare with."""
import ctypes as C
import os

import numpy as np
import pytest

from paper_2402_14139_amd import binding as nf
from tests import mx_ref, pointwise_ref

GOOD, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(nf.LIB_PATH):
        from paper_2402_14139_amd import build
        build.build()
    return nf.lib()


def _desc(**kw):
    return nf.LinearDesc(**{**dict(dtype=nf.NF_BF16, K=2048, N=64, act=nf.NF_ACT_GELU), **kw})


@pytest.mark.parametrize("desc,M,status", [
    (dict(dtype=3), 4, nf.NF_ERR_BAD_DESC), (dict(act=4), 4, nf.NF_ERR_BAD_DESC), (dict(K=0), 4, nf.NF_ERR_BAD_DESC),
    (dict(N=-1), 4, nf.NF_ERR_BAD_DESC), (dict(), 0, nf.NF_ERR_BAD_DESC), (dict(), -5, nf.NF_ERR_BAD_DESC),
    (dict(K=(1 << 24) + 1), 4, nf.NF_ERR_UNSUPPORTED), (dict(N=(1 << 20) + 1), 4, nf.NF_ERR_UNSUPPORTED),
    (dict(), (1 << 31) - 1, nf.NF_ERR_UNSUPPORTED), (dict(N=1 << 20), 1 << 20, nf.NF_ERR_UNSUPPORTED)])
def test_descriptors(L, desc, M, status):
    d, out = C.byref(_desc(**desc)), C.c_size_t()
    assert L.nf_mx_product_workspace_bytes(d, M, C.byref(out)) == L.nf_mx_linear_workspace_bytes(d, M, C.byref(out)) == status
    assert L.nf_mx_product(d, M, *[GOOD] * 8, 1 << 60, None) == status
    assert L.nf_mx_linear_fwd(d, M, GOOD, GOOD, GOOD, GOOD, GOOD, None, GOOD, GOOD, GOOD, 1 << 60, None) == status


def test_product_refusals(L):
    d, M = C.byref(_desc()), 64
    need = nf.nf_mx_product_workspace_bytes(_desc(), M)
    assert need > 0
    assert L.nf_mx_product_workspace_bytes(d, M, None) == L.nf_mx_product_workspace_bytes(None, M, C.byref(C.c_size_t())) == nf.NF_ERR_NULL
    names = ("a", "as", "b", "bs", "bias", "r", "y")
    call = lambda ws=GOOD, n=need, **kw: L.nf_mx_product(d, M, *[kw.get(k, GOOD) for k in names], ws, n, None)  # noqa: E731
    for k in ("a", "as", "b", "bs", "y"):
        assert call(**{k: None}) == nf.NF_ERR_NULL
    for k in names:
        assert call(**{k: ODD}) == nf.NF_ERR_BAD_DESC
    assert call(ws=None) == call(ws=0x10010) == call(n=need - 1) == nf.NF_ERR_WORKSPACE
    assert L.nf_mx_product(None, M, *[GOOD] * 8, need, None) == nf.NF_ERR_NULL


def test_linear_refusals(L):
    d, M = C.byref(_desc()), 64
    need = nf.nf_mx_linear_workspace_bytes(_desc(), M)
    assert need >= nf.nf_mx_product_workspace_bytes(_desc(), M) + M * (1024 + 64)
    assert L.nf_mx_linear_workspace_bytes(d, M, None) == L.nf_mx_linear_workspace_bytes(None, M, C.byref(C.c_size_t())) == nf.NF_ERR_NULL
    names = ("x", "W", "Ws", "b", "r", "drop", "y", "z")
    call = lambda ws=GOOD, n=need, **kw: L.nf_mx_linear_fwd(d, M, *[kw.get(k, None if k == "drop" else GOOD) for k in names], ws, n, None)  # noqa: E731
    for k in ("x", "W", "Ws", "y"):
        assert call(**{k: None}) == nf.NF_ERR_NULL
    for k in ("x", "W", "Ws", "b", "r", "y", "z"):
        assert call(**{k: ODD}) == nf.NF_ERR_BAD_DESC
    assert call(ws=None) == call(ws=0x10010) == call(n=need - 1) == nf.NF_ERR_WORKSPACE
    for p in (-0.1, 1.0, float("nan")):
        assert call(drop=C.byref(nf.DropoutDesc(p, 1, 2))) == nf.NF_ERR_BAD_DESC
    assert nf.nf_mx_linear_workspace_bytes(_desc(), 32) == 0   # quantised within the product's launch


def test_quantise_refusals(L):
    names = ("x", "codes", "scales", "codes_t", "scales_t")
    call = lambda dt=nf.NF_F32, rows=8, cols=40, **kw: L.nf_mx_quantise(dt, rows, cols, *[kw.get(k, GOOD) for k in names], None)  # noqa: E731
    for k in names:
        assert call(**{k: None}) == nf.NF_ERR_NULL and call(**{k: ODD}) == nf.NF_ERR_BAD_DESC
    assert call(codes=None, scales=None, codes_t=None, scales_t=None) == nf.NF_ERR_NULL
    assert call(dt=3) == call(dt=-1) == call(rows=0) == call(cols=0) == call(rows=-1) == call(cols=-7) == nf.NF_ERR_BAD_DESC
    assert call(rows=1 << 43, cols=3) == call(rows=1, cols=1 << 45) == call(rows=1 << 62, cols=1 << 62) == nf.NF_ERR_UNSUPPORTED
    assert call(rows=1, cols=1 << 40) == nf.NF_ERR_UNSUPPORTED   # more tiles than a grid has
    # 2^32 groups by rows, 2^24 tiles by columns: more threads than a launch has
    assert call(rows=1 << 32, cols=1, codes_t=None, scales_t=None) == call(rows=1 << 31, cols=1) == call(rows=1 << 12, cols=1 << 25) == nf.NF_ERR_UNSUPPORTED


def test_reference_against_the_caches():
    """The vectorised reference and the cache's: the same exponents and values, edges and powers of two among them."""
    g = np.random.RandomState(3)
    x = (g.randn(6, 100) * 2.0 ** g.randint(-20, 20, (6, 100))).astype(np.float32)
    x[0, :32], x[1, :32] = 0, np.float32(2.0 ** -140)
    x[2, :4], x[3, 5], x[4, 40], x[5, 99] = [6, 0.25, 0.75, 5], np.inf, np.nan, 3e38
    x[2, 4:32] = 0
    code, byte, v = mx_ref.quantise(x)
    wb, wv = pointwise_ref.quantise(nf.NF_Q_E2M1, x.astype(np.float64))
    assert (byte == wb).all() and np.array_equal(v, wv, equal_nan=True)
    assert list(code[2, :4]) == [7, 0, 2, 6] and byte[3, 0] == 255 and byte[0, 0] == 0
    packed, ex = mx_ref.pack(code, byte, (64, 16))
    assert np.array_equal(mx_ref.unpack(packed, 100), code) and (packed[:, 50:] == 255).all() and (ex[:, 4:] == 255).all()
