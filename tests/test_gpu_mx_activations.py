"""Activations behind products of 4-bit operands: the digits, and the bits, of those behind `nf_linear_fwd`, in every kernel that has an epilogue."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests.pointwise_ref import ACTS, DT, HALF, TINY, TYPES
from tests.test_gpu_activations import U, UNDER, check, definition, line, terms
from tests.test_gpu_pointwise import workspace

pytestmark = pytest.mark.gpu

# rows and terms that reach the few rows' kernel, tiles of 64, parts of sums, tiles of 128 with short and long sums, tiles of 256
SHAPES = [(1, 32), (20, 32), (40, 32), (40, 2100), (2000, 32), (2000, 800), (4000, 40000)]


def biases_alone(t, name, M, K, z):
    """Sums of nothing but a bias."""
    N = z.numel()
    a, b = (tuple(torch.zeros(r, s, dtype=torch.uint8, device="cuda") for s in nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, K)) for r in (M, N))
    d = nf.LinearDesc(dtype=DT[t], K=K, N=N, act=ACTS.index(name))
    y = torch.empty(M, N, dtype=TYPES[t], device="cuda")
    nf.nf_mx_product(d, M, *a, *b, z.float().cuda(), None, y, workspace(nf.nf_mx_product_workspace_bytes(d, M)))
    return y


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("M,K", SHAPES)
def test_digits(t, name, M, K):
    """The tolerance of the linear layer's activations: relative to the tail, not to the argument."""
    z = line(t)
    got = biases_alone(t, name, M, K, z)
    assert torch.equal(got, got[:1].expand(M, -1))
    Z = z.double()
    want = definition(name, Z)[0]
    _, r, Q, _, a = terms(t, Z)
    if name == "silu":     # e^-z, the sum, the quotient, the product
        tol = torch.nan_to_num(want.abs(), posinf=0.0) * U * (r * 2 + 3 if t == "f32" else r * (2 * a + 2) + 4) + UNDER
    else:                  # the fit; the bell's argument and value, t, the polynomial and two products; the final sum
        fit, arg, low = (1.6e-8, 0.5, UNDER) if t == "f32" else (2.1e-6, 1.5, 4e-18)
        tol = a * Q * (fit + (14 + arg * a * a) * U) + U * torch.nan_to_num(want.abs(), posinf=0.0) + low
    tol = tol + HALF[t] * (torch.nan_to_num(want.abs(), posinf=0.0) + tol) * (t != "f32") + TINY[t]
    check(name, got[0].double().cpu(), want, tol, z)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M,K", SHAPES[:5])
def test_the_linear_layers_bits(t, name, M, K):
    z = line(t)
    N = z.numel()
    d = nf.LinearDesc(dtype=DT[t], K=8, N=N, act=ACTS.index(name))
    y = torch.empty(M, N, dtype=TYPES[t], device="cuda")
    x, W = torch.zeros(M, 8, dtype=TYPES[t], device="cuda"), torch.zeros(N, 8, dtype=TYPES[t], device="cuda")
    nf.nf_linear_fwd(d, M, x, W, z.float().cuda(), None, None, y, None, workspace(max(1, nf.nf_linear_workspace_bytes(d, M))))
    assert torch.equal(biases_alone(t, name, M, K, z), y)
