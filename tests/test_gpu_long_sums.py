"""Long sums on the GPU, held by bounds that a part left out exceeds."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import long_sums as ls
from tests import mx_ref
from tests.pointwise_ref import DT, TYPES
from tests.test_gpu_pointwise import Out, close, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("M,C", ls.NORMS)
def test_norms(t, M, C):
    x, dy, mean, rstd = ls.norm_case(M, C, TYPES[t])
    d = nf.LayerNormDesc(dtype=DT[t], C=C, eps=1e-5)
    dx, dgamma, dbeta = torch.empty(M, C, dtype=TYPES[t], device="cuda"), Out(C), Out(C)
    nf.nf_layernorm_bwd(d, M, dy.cuda(), x.cuda(), None, mean.cuda(), rstd.cuda(), None, dx, dgamma.t, dbeta.t,
                        workspace(nf.nf_layernorm_workspace_bytes(d, M)))
    want_g, want_b, tol_g, tol_b = ls.norm_sums(x, dy, mean, rstd)
    close("dgamma", dgamma.cpu(), want_g, tol_g)
    close("dbeta", dbeta.cpu(), want_b, tol_b)


@pytest.mark.parametrize("M,K,N", ls.PRODUCTS)
def test_products(M, K, N):
    (qa, ea, A), (qb, eb, B) = ls.four_bits(M, K, N)
    strides = nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, K)
    a, b = (tuple(p.cuda() for p in mx_ref.pack(q, e, strides)) for q, e in ((qa, ea), (qb, eb)))
    d = nf.LinearDesc(dtype=nf.NF_F32, K=K, N=N, act=0)
    y = Out(M, N)
    nf.nf_mx_product(d, M, *a, *b, None, None, y.t, workspace(nf.nf_mx_product_workspace_bytes(d, M)))
    close("y", y.cpu(), *ls.product(A, B))
