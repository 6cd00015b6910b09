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


def test_group_norm_of_more_workgroups_than_one_axis_takes():
    """2048 slabs to an image of one pixel and 32769 images: 2^32 threads and more.  Groups of two channels: the results are
    +-h / sqrt(h^2 + eps) with h half their distance, dx next to nothing but for the residue of eps."""
    B, Ch, G, eps = (1 << 15) + 1, 1 << 16, 1 << 15, 1.0
    d = nf.GroupNormDesc(dtype=nf.NF_F32, C=Ch, G=G, act=nf.NF_ACT_NONE, HW=1, eps=eps)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(B, Ch, generator=g, device="cuda")
    gamma, beta = torch.ones(Ch, device="cuda"), torch.zeros(Ch, device="cuda")
    new = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    y, mean, rstd = new(B, Ch), new(B, G), new(B, G)
    ws = torch.empty(nf.nf_groupnorm_workspace_bytes(d, B), dtype=torch.uint8, device="cuda")
    nf.nf_groupnorm_fwd(d, B, x, gamma, beta, y, mean, rstd, ws)
    dy, dx, dg, db = torch.randn(B, Ch, generator=g, device="cuda"), new(B, Ch), new(Ch), new(Ch)
    nf.nf_groupnorm_bwd(d, B, dy, x, gamma, beta, mean, rstd, dx, dg, db, ws)
    sums = [torch.zeros(Ch, dtype=torch.float64, device="cuda") for _ in range(4)]
    for i in range(0, B, 2048):
        X, D = (v[i:i + 2048].double().view(-1, G, 2) for v in (x, dy))
        mu = X.mean(2)
        h = (X[..., 0] - X[..., 1]) / 2
        rs = (h * h + eps).rsqrt()
        xh = torch.stack([h * rs, -h * rs], 2)
        top = X.abs().amax(2, keepdim=True)
        tol = 16 * SUM * (1 + top)     # a dozen roundings of terms no larger than top, and deviations of 1 at the least
        assert ((y[i:i + 2048].double().view_as(X) - xh).abs() <= tol).all(), i
        assert ((mean[i:i + 2048].double() - mu).abs() <= tol[..., 0]).all() and ((rstd[i:i + 2048].double() - rs).abs() <= 16 * SUM * (1 + top[..., 0])).all()
        avg, avx = D.mean(2, keepdim=True), (D * xh).mean(2, keepdim=True)
        want = rs[..., None] * (D - avg - xh * avx)
        assert ((dx[i:i + 2048].double().view_as(X) - want).abs() <= 2 * tol * (1 + D.abs().amax(2, keepdim=True)) * (1 + top)).all(), i
        for s, v in zip(sums, (D * xh, D, (D * xh).abs() + 16 * D.abs() * (1 + top), D.abs())):
            s += v.reshape(-1, Ch).sum(0)
    # sums over images in trees: some 250 roundings of the terms, whose own roundings stand in the magnitudes
    assert ((dg.double() - sums[0]).abs() <= 250 * SUM * sums[2]).all() and ((db.double() - sums[1]).abs() <= 250 * SUM * sums[3]).all()
