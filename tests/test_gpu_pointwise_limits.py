"""Sizes at the ends of the admitted ranges, where a launch's grid would pass its limits."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests.pointwise_ref import DT, HALF, SUM, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,K,N", [("f32", 3, 1), ("bf16", 1, 3), ("f16", 7, 1), ("bf16", 1, 1)])
@pytest.mark.parametrize("M", [(65535 << 6) - 1, (65536 << 6) + 100])
def test_linear_of_few_weights_and_many_rows(t, K, N, M):
    """Weights of less than 16 bytes: a workgroup to 64 rows, more than 65535 of them."""
    T = TYPES[t]
    g = torch.Generator(device="cuda").manual_seed(K + N)
    x, r = torch.randn(M, K, generator=g, device="cuda").to(T), torch.randn(M, N, generator=g, device="cuda").to(T)
    W, b = torch.randn(N, K, generator=g, device="cuda").to(T), torch.randn(N, generator=g, device="cuda")
    d = nf.LinearDesc(dtype=DT[t], K=K, N=N, act=nf.NF_ACT_RELU)
    assert nf.nf_linear_fwd_workspace_bytes(d, M) == 0
    out = torch.full((M + 64, N), 5.0, dtype=T, device="cuda")
    nf.nf_linear_fwd(d, M, x, W, b, r, None, out, None, None)
    Z = (x.double()[:, None, :] * W.double()[None]).sum(2) + b.double()
    err = (K + 3) * SUM * ((x.double()[:, None, :] * W.double()[None]).abs().sum(2) + b.double().abs() + r.double().abs())
    Y = Z.clamp_min(0) + r.double()
    assert ((out[:M].double() - Y).abs() <= err + HALF[t] * (Y.abs() + err) + 2.0 ** -25).all()
    assert (out[M:] == 5).all()
