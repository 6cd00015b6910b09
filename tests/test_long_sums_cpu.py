"""The bounds of the long sums' tests: results without a part of the terms, or without any, lie outside."""
import pytest
import torch

from tests import long_sums as ls


@pytest.mark.parametrize("M,C", ls.NORMS)
def test_norms(M, C):
    x, dy, mean, rstd = ls.norm_case(M, C, torch.bfloat16)
    dgamma, dbeta, tol_g, tol_b = ls.norm_sums(x, dy, mean, rstd)
    assert (dgamma.abs() > 10 * tol_g).all() and (dbeta.abs() > 10 * tol_b).all()   # none, or a part of a tenth
    rows = max(M // 1024, 16)   # a workgroup's
    for first in (0, M // 2, M - rows):
        xh = (x[first:first + rows].double() - mean[first:first + rows].double()[:, None]) * rstd[first:first + rows].double()[:, None]
        d = dy[first:first + rows].double()
        assert ((d * xh).sum(0).abs() > tol_g).float().mean() > 0.9 and (d.sum(0).abs() > tol_b).float().mean() > 0.9


@pytest.mark.parametrize("M,K,N", ls.PRODUCTS)
def test_products(M, K, N):
    (_, _, A), (_, _, B) = ls.four_bits(M, K, N)
    want, tol = ls.product(A, B)
    assert (want.abs() > tol).double().mean() > 0.95
    for first in (0, K // 2, K - 256):   # a step of the sum
        part = A[:, first:first + 256] @ B[:, first:first + 256].t()
        assert (part.abs() > tol).double().mean() > 0.5
