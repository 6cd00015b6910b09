"""Layer norm without a GPU: refusals, sizes, and the reference the GPU tests compare with."""
import ctypes as C
import os

import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import layer_norm_ref as ref

GOOD, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(nf.LIB_PATH):
        from paper_2402_14139_amd import build
        build.build()
    return nf.lib()


def _desc(**kw):
    return nf.LayerNormDesc(**{**dict(dtype=nf.NF_BF16, C=512, eps=1e-5), **kw})


@pytest.mark.parametrize("desc,M,status", [
    (dict(dtype=3), 2, nf.NF_ERR_BAD_DESC), (dict(dtype=-1), 2, nf.NF_ERR_BAD_DESC), (dict(C=0), 2, nf.NF_ERR_BAD_DESC),
    (dict(C=-4), 2, nf.NF_ERR_BAD_DESC), (dict(eps=-1e-9), 2, nf.NF_ERR_BAD_DESC), (dict(eps=float("nan")), 2, nf.NF_ERR_BAD_DESC),
    (dict(), 0, nf.NF_ERR_BAD_DESC), (dict(), -3, nf.NF_ERR_BAD_DESC), (dict(C=(1 << 16) + 1), 2, nf.NF_ERR_UNSUPPORTED),
    (dict(), 1 << 40, nf.NF_ERR_UNSUPPORTED)])
def test_descriptors(L, desc, M, status):
    d, out = C.byref(_desc(**desc)), C.c_size_t()
    assert L.nf_layernorm_workspace_bytes(d, M, C.byref(out)) == status
    assert L.nf_layernorm_fwd(d, M, *[GOOD] * 6, None) == status
    assert L.nf_layernorm_bwd(d, M, *[GOOD] * 10, 1 << 60, None) == status


def test_refusals(L):
    d, M = C.byref(_desc()), 5000
    need = nf.nf_layernorm_workspace_bytes(_desc(), M)
    assert need > 0
    assert L.nf_layernorm_workspace_bytes(None, M, C.byref(C.c_size_t())) == L.nf_layernorm_workspace_bytes(d, M, None) == nf.NF_ERR_NULL
    fwd = lambda x=GOOD, gamma=GOOD, beta=GOOD, y=GOOD, mean=GOOD, rstd=GOOD: L.nf_layernorm_fwd(d, M, x, gamma, beta, y, mean, rstd, None)  # noqa: E731
    assert fwd(x=None) == fwd(y=None) == fwd(mean=None) == fwd(rstd=None) == nf.NF_ERR_NULL
    for k in ("x", "gamma", "beta", "y", "mean", "rstd"):
        assert fwd(**{k: ODD}) == nf.NF_ERR_BAD_DESC
    def bwd(dy=GOOD, x=GOOD, gamma=GOOD, mean=GOOD, rstd=GOOD, dr=GOOD, dx=GOOD, dgamma=GOOD, dbeta=GOOD, ws=GOOD, n=need):
        return L.nf_layernorm_bwd(d, M, dy, x, gamma, mean, rstd, dr, dx, dgamma, dbeta, ws, n, None)
    assert bwd(dy=None) == bwd(x=None) == bwd(mean=None) == bwd(rstd=None) == bwd(dx=None, dgamma=None, dbeta=None) == nf.NF_ERR_NULL
    for k in ("dy", "x", "gamma", "mean", "rstd", "dr", "dx", "dgamma", "dbeta"):
        assert bwd(**{k: ODD}) == nf.NF_ERR_BAD_DESC
    assert bwd(ws=None) == bwd(ws=0x10010) == bwd(n=need - 1) == bwd(dgamma=None, ws=None) == bwd(dbeta=None, n=0) == nf.NF_ERR_WORKSPACE


def test_reference_gradient_against_differences():
    g = torch.Generator().manual_seed(4)
    rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, gamma, beta, w, eps = rn(3, 7), rn(7), rn(7), rn(3, 7), 1e-3
    f = lambda x, ga, be: (ref.forward(x, ga, be, eps)[0] * w).sum()  # noqa: E731
    _, mean, rstd = ref.forward(x, gamma, beta, eps)
    h = 1e-6
    for k, (t, grad) in enumerate(zip((x, gamma, beta), ref.gradients(w, x, gamma, mean, rstd))):
        for i in range(t.numel()):
            d = torch.zeros(t.numel(), dtype=torch.float64)
            d[i] = h
            up, down = [x, gamma, beta], [x, gamma, beta]
            up[k], down[k] = t + d.view(t.shape), t - d.view(t.shape)
            assert abs((f(*up) - f(*down)) / (2 * h) - grad.reshape(-1)[i]) < 1e-6
