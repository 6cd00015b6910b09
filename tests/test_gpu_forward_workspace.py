"""Forward calls run in the workspace that the forward alone wants, often none, and write nothing behind it."""
import ctypes as C

import pytest
import torch

from paper_2402_14139_amd import binding as nf

GOOD = 0x10000
LINEAR = [(2000, 64, 128), (4096, 512, 512), (64, 2048, 64), (300, 520, 256), (100, 1000, 65)]
NORMS = [(3, 64, 16, 4), (2, 1024, 72, 6), (1, 700, 1536, 3), (2, 300, 515, 1), (2, 4096, 512, 8)]


def band(n):
    """n bytes, and 4096 behind them that nothing may write"""
    ws = torch.full((n + 4096,), 165, dtype=torch.uint8, device="cuda")
    return ws, (ws[:n] if n else None)


@pytest.mark.parametrize("dtype", [nf.NF_F32, nf.NF_BF16])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_sizes_of_the_linear_layer(dtype, M, K, N):
    d = nf.LinearDesc(dtype=dtype, K=K, N=N, act=0)
    fwd = nf.nf_linear_fwd_workspace_bytes(d, M)
    assert 0 <= fwd <= nf.nf_linear_workspace_bytes(d, M)
    if fwd:
        assert nf.lib().nf_linear_fwd(C.byref(d), M, GOOD, GOOD, None, None, None, GOOD, None, GOOD, fwd - 1, None) == nf.NF_ERR_WORKSPACE


@pytest.mark.parametrize("dtype", [nf.NF_F32, nf.NF_BF16])
@pytest.mark.parametrize("B,HW,Ch,G", NORMS)
def test_sizes_of_group_norm(dtype, B, HW, Ch, G):
    d = nf.GroupNormDesc(dtype=dtype, C=Ch, G=G, act=0, HW=HW, eps=1e-5)
    fwd = nf.nf_groupnorm_fwd_workspace_bytes(d, B)
    assert 0 <= fwd < nf.nf_groupnorm_workspace_bytes(d, B)
    if fwd:
        assert nf.lib().nf_groupnorm_fwd(C.byref(d), B, *[GOOD] * 6, GOOD, fwd - 1, None) == nf.NF_ERR_WORKSPACE


def test_refusals():
    out, L = C.c_size_t(), nf.lib()
    d, n = nf.LinearDesc(dtype=0, K=8, N=8, act=0), nf.GroupNormDesc(dtype=0, C=8, G=2, act=0, HW=4, eps=1e-5)
    assert L.nf_linear_fwd_workspace_bytes(None, 4, C.byref(out)) == L.nf_groupnorm_fwd_workspace_bytes(None, 4, C.byref(out)) == nf.NF_ERR_NULL
    assert L.nf_linear_fwd_workspace_bytes(C.byref(d), 4, None) == L.nf_groupnorm_fwd_workspace_bytes(C.byref(n), 4, None) == nf.NF_ERR_NULL
    assert L.nf_linear_fwd_workspace_bytes(C.byref(d), 0, C.byref(out)) == nf.NF_ERR_BAD_DESC
    assert L.nf_groupnorm_fwd_workspace_bytes(C.byref(n), 0, C.byref(out)) == nf.NF_ERR_BAD_DESC


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T", [(nf.NF_F32, torch.float32), (nf.NF_BF16, torch.bfloat16)])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_linear(dtype, T, M, K, N):
    g = torch.Generator().manual_seed(M)
    x, W, b = torch.randn(M, K, generator=g).to(T).cuda(), torch.randn(N, K, generator=g).to(T).cuda(), torch.randn(N, generator=g).cuda()
    d = nf.LinearDesc(dtype=dtype, K=K, N=N, act=nf.NF_ACT_SILU)
    own, all_ = nf.nf_linear_fwd_workspace_bytes(d, M), nf.nf_linear_workspace_bytes(d, M)
    want, got = (torch.empty(M, N, dtype=T, device="cuda") for _ in range(2))
    nf.nf_linear_fwd(d, M, x, W, b, None, None, want, None, band(all_)[0])
    whole, ws = band(own)
    nf.nf_linear_fwd(d, M, x, W, b, None, None, got, None, ws)
    assert torch.equal(got, want) and (whole[own:] == 165).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T", [(nf.NF_F32, torch.float32), (nf.NF_BF16, torch.bfloat16)])
@pytest.mark.parametrize("B,HW,Ch,G", NORMS)
def test_group_norm(dtype, T, B, HW, Ch, G):
    x = torch.randn(B, HW, Ch, generator=torch.Generator().manual_seed(HW)).to(T).cuda()
    gamma, beta = torch.ones(Ch, device="cuda"), torch.zeros(Ch, device="cuda")
    d = nf.GroupNormDesc(dtype=dtype, C=Ch, G=G, act=nf.NF_ACT_RELU, HW=HW, eps=1e-5)
    own, all_ = nf.nf_groupnorm_fwd_workspace_bytes(d, B), nf.nf_groupnorm_workspace_bytes(d, B)
    whole, ws = band(own)
    want, got = ([torch.empty_like(x), torch.empty(B, G, device="cuda"), torch.empty(B, G, device="cuda")] for _ in range(2))
    nf.nf_groupnorm_fwd(d, B, x, gamma, beta, *want, band(all_)[0])
    nf.nf_groupnorm_fwd(d, B, x, gamma, beta, *got, ws)
    assert all(torch.equal(u, v) for u, v in zip(got, want)) and (whole[own:] == 165).all()
