"""Pointwise layers and the quantised cache without a GPU: refusals, sizes, and the reference the GPU tests compare with."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import pointwise_ref as ref

GOOD, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(nf.LIB_PATH):
        from paper_2402_14139_amd import build
        build.build()
    return nf.lib()


def test_philox_known_answers():
    """The generator's published vectors, through both forms of the reference."""
    assert ref.philox([0] * 4, [0, 0]) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert ref.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    seed, step = 0x1234567890ABCDEF, 0xFEDCBA0987654321
    T = 0.3
    k = ref.keep_scale(2, 13, T, seed, step)
    for row in range(2):
        for col in range(13):
            w = ref.philox([row * 2 + col // 8, 0, step & 0xFFFFFFFF, step >> 32], [seed & 0xFFFFFFFF, seed >> 32])
            u = w[col % 8 // 2] >> 16 * (col % 2) & 0xFFFF
            assert k[row, col] == (65536 / (65536 - 19661) if u >= 19661 else 0)


def test_codebooks():
    assert ref.codebook(nf.NF_Q_E2M1) == [0, .5, 1, 1.5, 2, 3, 4, 6]
    e4m3 = ref.codebook(nf.NF_Q_E4M3)
    assert e4m3[-1] == 448 and e4m3[1] == 2.0 ** -9 and e4m3[8] == 2.0 ** -6


@pytest.mark.parametrize("name", ref.ACTS)
def test_reference_slopes_against_differences(name):
    z = torch.linspace(-6, 6, 241, dtype=torch.float64) + 0.013
    h = 1e-5
    assert torch.allclose(ref.slope(name, z), (ref.act(name, z + h) - ref.act(name, z - h)) / (2 * h), atol=1e-9)


@pytest.mark.parametrize("name", ref.ACTS)
def test_reference_group_norm_gradient_against_differences(name):
    g = torch.Generator().manual_seed(5)
    x, w = torch.randn(2, 5, 6, generator=g, dtype=torch.float64), torch.randn(2, 5, 6, generator=g, dtype=torch.float64)
    gamma, beta = torch.randn(6, generator=g, dtype=torch.float64), torch.randn(6, generator=g, dtype=torch.float64)
    f = lambda x, ga, be: (ref.group_norm(x, ga, be, 2, 1e-5, name)[0] * w).sum()  # noqa: E731
    _, mean, rstd = ref.group_norm(x, gamma, beta, 2, 1e-5, name)
    grads = ref.group_norm_grad(w, x, gamma, beta, mean, rstd, name)[:3]
    h = 1e-6
    for k, t in enumerate((x, gamma, beta)):
        for i in range(t.numel()):
            d = torch.zeros_like(t).reshape(-1)
            d[i] = h
            d = d.reshape(t.shape)
            up, down = [x, gamma, beta], [x, gamma, beta]
            up[k], down[k] = t + d, t - d
            assert abs((f(*up) - f(*down)) / (2 * h) - grads[k].reshape(-1)[i]) < 1e-6


def test_row_bytes(L):
    assert nf.nf_qcache_row_bytes(nf.NF_Q_INT8, 1) == (16, 16)
    assert nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, 33) == (32, 16)
    assert nf.nf_qcache_row_bytes(nf.NF_Q_E4M3, 16384) == (16384, 512)
    c = C.c_size_t()
    assert L.nf_qcache_row_bytes(3, 8, C.byref(c), C.byref(c)) == nf.NF_ERR_BAD_DESC
    assert L.nf_qcache_row_bytes(0, 0, C.byref(c), C.byref(c)) == nf.NF_ERR_BAD_DESC
    assert L.nf_qcache_row_bytes(0, 8, None, C.byref(c)) == nf.NF_ERR_NULL


def _linear(**kw):
    return nf.LinearDesc(**{**dict(dtype=nf.NF_BF16, K=64, N=64, act=nf.NF_ACT_GELU), **kw})


def _norm(**kw):
    return nf.GroupNormDesc(**{**dict(dtype=nf.NF_F32, C=64, G=8, act=0, HW=16, eps=1e-5), **kw})


@pytest.mark.parametrize("desc,M,status", [
    (dict(dtype=3), 4, nf.NF_ERR_BAD_DESC), (dict(act=4), 4, nf.NF_ERR_BAD_DESC), (dict(K=0), 4, nf.NF_ERR_BAD_DESC),
    (dict(N=-1), 4, nf.NF_ERR_BAD_DESC), (dict(), 0, nf.NF_ERR_BAD_DESC), (dict(), -5, nf.NF_ERR_BAD_DESC),
    (dict(K=(1 << 20) + 1), 4, nf.NF_ERR_UNSUPPORTED), (dict(), (1 << 31) - 1, nf.NF_ERR_UNSUPPORTED)])
def test_linear_descriptors(L, desc, M, status):
    out = C.c_size_t()
    d = _linear(**desc)
    assert L.nf_linear_workspace_bytes(C.byref(d), M, C.byref(out)) == status
    assert L.nf_linear_fwd(C.byref(d), M, GOOD, GOOD, GOOD, GOOD, None, GOOD, GOOD, GOOD, 1 << 40, None) == status
    assert L.nf_linear_bwd_epilogue(C.byref(d), M, GOOD, GOOD, None, GOOD, GOOD, GOOD, 1 << 40, None) == status
    assert L.nf_linear_bwd(C.byref(d), M, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 1 << 40, None) == status


def test_linear_refusals(L):
    d, M = C.byref(_linear(K=2048, N=64)), 64
    need = nf.nf_linear_workspace_bytes(_linear(K=2048, N=64), M)
    assert need > 0
    fwd = lambda x=GOOD, W=GOOD, b=GOOD, r=GOOD, drop=None, y=GOOD, z=GOOD, ws=GOOD, n=need: \
        L.nf_linear_fwd(d, M, x, W, b, r, drop, y, z, ws, n, None)  # noqa: E731
    assert fwd(x=None) == fwd(W=None) == fwd(y=None) == nf.NF_ERR_NULL
    for k in ("x", "W", "b", "r", "y", "z"):
        assert fwd(**{k: ODD}) == nf.NF_ERR_BAD_DESC
    assert fwd(ws=None) == fwd(ws=0x10010) == fwd(n=need - 1) == nf.NF_ERR_WORKSPACE
    for p in (-0.1, 1.0, 0.99999999, float("nan")):
        assert fwd(drop=C.byref(nf.DropoutDesc(p, 1, 2))) == nf.NF_ERR_BAD_DESC
    epi = lambda dy=GOOD, z=GOOD, dz=GOOD, db=GOOD, ws=GOOD: L.nf_linear_bwd_epilogue(d, M, dy, z, None, dz, db, ws, need, None)  # noqa: E731
    assert epi(dy=None) == epi(z=None) == epi(dz=None) == nf.NF_ERR_NULL
    assert epi(db=ODD) == nf.NF_ERR_BAD_DESC and epi(ws=None) == nf.NF_ERR_WORKSPACE
    bwd = lambda dz=GOOD, x=GOOD, W=GOOD, dx=GOOD, dW=GOOD, ws=GOOD: L.nf_linear_bwd(d, M, dz, x, W, dx, dW, ws, need, None)  # noqa: E731
    assert bwd(dz=None) == bwd(dx=None, dW=None) == bwd(W=None) == bwd(x=None) == nf.NF_ERR_NULL
    assert bwd(dW=ODD) == nf.NF_ERR_BAD_DESC and bwd(ws=None) == nf.NF_ERR_WORKSPACE
    assert L.nf_linear_fwd(None, M, GOOD, GOOD, GOOD, GOOD, None, GOOD, GOOD, GOOD, need, None) == nf.NF_ERR_NULL
    assert L.nf_linear_workspace_bytes(d, M, None) == nf.NF_ERR_NULL


@pytest.mark.parametrize("desc,B,status", [
    (dict(dtype=-1), 2, nf.NF_ERR_BAD_DESC), (dict(act=9), 2, nf.NF_ERR_BAD_DESC), (dict(G=7), 2, nf.NF_ERR_BAD_DESC),
    (dict(HW=0), 2, nf.NF_ERR_BAD_DESC), (dict(eps=-1.0), 2, nf.NF_ERR_BAD_DESC), (dict(eps=float("nan")), 2, nf.NF_ERR_BAD_DESC),
    (dict(), 0, nf.NF_ERR_BAD_DESC), (dict(), 65536, nf.NF_ERR_UNSUPPORTED), (dict(C=4096, G=1), 2, nf.NF_ERR_UNSUPPORTED),
    (dict(HW=1 << 24), 2, nf.NF_ERR_UNSUPPORTED), (dict(C=1 << 17, G=1 << 17), 2, nf.NF_ERR_UNSUPPORTED)])
def test_group_norm_descriptors(L, desc, B, status):
    d, out = C.byref(_norm(**desc)), C.c_size_t()
    assert L.nf_groupnorm_workspace_bytes(d, B, C.byref(out)) == status
    assert L.nf_groupnorm_fwd(d, B, *[GOOD] * 7, 1 << 40, None) == status
    assert L.nf_groupnorm_bwd(d, B, *[GOOD] * 10, 1 << 40, None) == status


def test_group_norm_refusals(L):
    d = C.byref(_norm())
    need = nf.nf_groupnorm_workspace_bytes(_norm(), 2)
    for k in range(6):
        a = [GOOD] * 6
        a[k] = None
        assert L.nf_groupnorm_fwd(d, 2, *a, GOOD, need, None) == nf.NF_ERR_NULL
        a[k] = ODD
        assert L.nf_groupnorm_fwd(d, 2, *a, GOOD, need, None) == nf.NF_ERR_BAD_DESC
    for k in range(9):
        a = [GOOD] * 9
        a[k] = None
        assert L.nf_groupnorm_bwd(d, 2, *a, GOOD, need, None) == nf.NF_ERR_NULL
        a[k] = ODD
        assert L.nf_groupnorm_bwd(d, 2, *a, GOOD, need, None) == nf.NF_ERR_BAD_DESC
    if need:
        assert L.nf_groupnorm_bwd(d, 2, *[GOOD] * 9, None, need, None) == nf.NF_ERR_WORKSPACE
        assert L.nf_groupnorm_bwd(d, 2, *[GOOD] * 9, GOOD, need - 1, None) == nf.NF_ERR_WORKSPACE


def test_dropout_refusals(L):
    d = C.byref(nf.DropoutDesc(0.5, 1, 2))
    assert L.nf_dropout_fwd(None, 0, 2, 2, GOOD, None, GOOD, None) == nf.NF_ERR_NULL
    assert L.nf_dropout_fwd(d, 0, 2, 2, None, None, GOOD, None) == nf.NF_ERR_NULL
    assert L.nf_dropout_bwd(d, 0, 2, 2, GOOD, None, None) == nf.NF_ERR_NULL
    assert L.nf_dropout_fwd(d, 5, 2, 2, GOOD, None, GOOD, None) == nf.NF_ERR_BAD_DESC
    assert L.nf_dropout_fwd(d, 0, 0, 2, GOOD, None, GOOD, None) == nf.NF_ERR_BAD_DESC
    assert L.nf_dropout_fwd(d, 0, 2, -1, GOOD, None, GOOD, None) == nf.NF_ERR_BAD_DESC
    assert L.nf_dropout_fwd(d, 0, 2, 2, GOOD, ODD, GOOD, None) == nf.NF_ERR_BAD_DESC
    assert L.nf_dropout_bwd(d, 0, 2, 2, ODD, GOOD, None) == nf.NF_ERR_BAD_DESC
    assert L.nf_dropout_fwd(d, 0, 2, 1 << 31, GOOD, None, GOOD, None) == nf.NF_ERR_UNSUPPORTED
    assert L.nf_dropout_fwd(d, 0, 1 << 60, 1 << 20, GOOD, None, GOOD, None) == nf.NF_ERR_UNSUPPORTED
    assert L.nf_dropout_bwd(C.byref(nf.DropoutDesc(1.0, 1, 2)), 0, 2, 2, GOOD, GOOD, None) == nf.NF_ERR_BAD_DESC


def test_qcache_refusals(L):
    w = lambda fmt=0, dt=0, codes=GOOD, scales=GOOD, lab=GOOD, cap=10, n=64, first=0, B=4, x=GOOD, labels=GOOD: \
        L.nf_qcache_write(fmt, dt, codes, scales, lab, cap, n, first, B, x, labels, None)  # noqa: E731
    assert w(codes=None) == w(scales=None) == w(x=None) == w(labels=None) == w(lab=None) == nf.NF_ERR_NULL
    assert w(fmt=3) == w(dt=3) == w(cap=0) == w(n=0) == w(B=0) == w(B=65536, cap=1 << 20) == nf.NF_ERR_BAD_DESC
    assert w(codes=ODD) == w(scales=ODD) == w(x=ODD) == nf.NF_ERR_BAD_DESC
    assert w(first=-1) == w(first=7) == nf.NF_ERR_CACHE_RANGE
    assert w(first=(1 << 63) - 1) == nf.NF_ERR_CACHE_RANGE
    assert w(n=1 << 40) == nf.NF_ERR_UNSUPPORTED
    r = lambda fmt=0, first=0, idx=None, B=4: L.nf_qcache_read(fmt, 0, GOOD, GOOD, GOOD, 10, 64, first, idx, B, GOOD, GOOD, None)  # noqa: E731
    assert r(first=7) == nf.NF_ERR_CACHE_RANGE and r(fmt=-1) == nf.NF_ERR_BAD_DESC and r(idx=GOOD, B=0) == nf.NF_ERR_BAD_DESC


def test_reference_quantiser_by_hand():
    x = np.zeros((1, 40))
    x[0, :4] = [6.0, 2.5, -0.25, 5.0]
    x[0, 32:36] = [13.0, 6.5, 1.0, np.nan]
    b, v = ref.quantise(nf.NF_Q_E2M1, x[:, :32])
    assert b[0, 0] == 127 and list(v[0, :4]) == [6, 2, 0, 4]
    b, v = ref.quantise(nf.NF_Q_E2M1, x)
    assert b[0, 1] == 255 and np.isnan(v[0, 32:]).all()
    x[0, 35] = 0
    b, v = ref.quantise(nf.NF_Q_E2M1, x)
    assert b[0, 1] == 129 and list(v[0, 32:35]) == [12, 6, 0]
