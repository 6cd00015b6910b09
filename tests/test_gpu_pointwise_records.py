"""Measurements of the pointwise layers (nf_prof_begin, nf_prof_begin_as_run): every kernel under its own name, what shares a launch
apart or under a name of its own, and the same results either way."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf

pytestmark = pytest.mark.gpu


def recorded(call, as_run):
    nf.nf_prof_begin_as_run() if as_run else nf.nf_prof_begin()
    try:
        call()
    finally:
        got = nf.nf_prof_end()
    torch.cuda.synchronize()
    assert all(r["ms"] > 0 for r in got)
    return {r["kernel"]: r["launches"] for r in got}


def test_linear_gradients():
    M, K, N = 5000, 64, 48
    g = torch.Generator().manual_seed(0)
    x, W, dz = (torch.randn(*s, generator=g).bfloat16().cuda() for s in ((M, K), (N, K), (M, N)))
    d = nf.LinearDesc(dtype=nf.NF_BF16, K=K, N=N, act=0)
    ws = torch.empty(nf.nf_linear_workspace_bytes(d, M), dtype=torch.uint8, device="cuda")
    out = [(torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(N, K, device="cuda")) for _ in range(3)]
    call = lambda o: nf.nf_linear_bwd(d, M, dz, x, W, *o, ws)  # noqa: E731
    call(out[0])
    assert recorded(lambda: call(out[1]), False) == {"linear_dx_64x64": 1, "linear_dw_64x64": 1, "linear_dw_finish": 1}
    assert recorded(lambda: call(out[2]), True) == {"linear_gradients_64_64": 1, "linear_dw_finish": 1}
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))


def test_both_gradients_in_parts():
    M, K, N = 2100, 72, 1600
    g = torch.Generator().manual_seed(0)
    x, W, dz = (torch.randn(*s, generator=g).cuda() for s in ((M, K), (N, K), (M, N)))
    d = nf.LinearDesc(dtype=nf.NF_F32, K=K, N=N, act=0)
    ws = torch.empty(nf.nf_linear_workspace_bytes(d, M), dtype=torch.uint8, device="cuda")
    out = [(torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")) for _ in range(2)]
    call = lambda o: nf.nf_linear_bwd(d, M, dz, x, W, *o, ws)  # noqa: E731
    assert recorded(lambda: call(out[0]), False) == {"linear_dx_64x64": 1, "linear_dw_64x64": 1, "linear_dx_finish": 1, "linear_dw_finish": 1}
    assert recorded(lambda: call(out[1]), True) == {"linear_gradients_64_64": 1, "linear_gradients_finish": 1}
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_forward_and_epilogue():
    M, K, N = 1000, 2048, 64
    x, W = torch.ones(M, K, dtype=torch.float16, device="cuda"), torch.ones(N, K, dtype=torch.float16, device="cuda")
    y, db = torch.empty(M, N, dtype=torch.float16, device="cuda"), torch.empty(N, device="cuda")
    d = nf.LinearDesc(dtype=nf.NF_F16, K=K, N=N, act=0)
    ws = torch.empty(nf.nf_linear_workspace_bytes(d, M), dtype=torch.uint8, device="cuda")
    assert recorded(lambda: nf.nf_linear_fwd(d, M, x, W, None, None, None, y, None, ws), False) == {"linear_fwd_64x64": 1, "linear_fwd_finish": 1}
    assert (y == 2048).all()
    assert recorded(lambda: nf.nf_linear_fwd(d, 1, x, W, None, None, None, y, None, ws), True) == {"linear_fwd_8_rows_long": 1}
    assert recorded(lambda: nf.nf_linear_bwd_epilogue(d, M, y, None, None, y.clone(), db, ws), False) == {"linear_bwd_epilogue": 1, "linear_bias_sums": 1}
    assert (db == 2048.0 * M).all()


def test_group_norm():
    B, HW, C, G = 3, 64, 16, 4
    x = torch.randn(B, HW, C, device="cuda")
    one, zero = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    d = nf.GroupNormDesc(dtype=nf.NF_F32, C=C, G=G, act=0, HW=HW, eps=1e-5)
    ws = torch.empty(nf.nf_groupnorm_workspace_bytes(d, B), dtype=torch.uint8, device="cuda")
    y, mean, rstd, dg, db = torch.empty_like(x), *(torch.empty(B, G, device="cuda") for _ in range(2)), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    assert recorded(lambda: nf.nf_groupnorm_fwd(d, B, x, one, zero, y, mean, rstd, ws), False) == {"groupnorm_fwd_few_64": 1}
    assert recorded(lambda: nf.nf_groupnorm_bwd(d, B, x, x, one, zero, mean, rstd, y, dg, db, ws), False) == {"groupnorm_bwd_few_64": 1, "groupnorm_bwd_sums": 1}
    d = nf.GroupNormDesc(dtype=nf.NF_F32, C=1536, G=3, act=0, HW=700, eps=1e-5)
    x = torch.randn(2, 700, 1536, device="cuda")
    one, zero = torch.ones(1536, device="cuda"), torch.zeros(1536, device="cuda")
    ws = torch.empty(nf.nf_groupnorm_workspace_bytes(d, 2), dtype=torch.uint8, device="cuda")
    y, mean, rstd, dg, db = torch.empty_like(x), *(torch.empty(2, 3, device="cuda") for _ in range(2)), torch.empty(1536, device="cuda"), torch.empty(1536, device="cuda")
    assert recorded(lambda: nf.nf_groupnorm_fwd(d, 2, x, one, zero, y, mean, rstd, ws), False) == {"groupnorm_fwd_stats": 1, "groupnorm_fwd_apply": 1}
    assert recorded(lambda: nf.nf_groupnorm_bwd(d, 2, x, x, one, zero, mean, rstd, y, dg, db, ws), False) == \
        {"groupnorm_bwd_stats": 1, "groupnorm_bwd_chunk_sums": 1, "groupnorm_bwd_apply": 1, "groupnorm_bwd_sums": 1}
