"""Activations and their slopes over the whole line, through the linear layer: large finite numbers and infinities, and errors that
count the roundings of each formula, by the type whose results they are.

u is half a step of fp32, relative.  The 16-bit types take e^v as a power of two of v log2 e (two roundings of the argument, which
weigh |v| of it, and one step) and 1 / v to one step."""
import math

import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import pointwise_ref as ref
from tests.pointwise_ref import ACTS, DT, HALF, TINY, TYPES

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
UNDER = 2e-36   # below it e^v has left fp32's normal numbers


def line(t):
    far = [18.3, 19.7, 40.0, 87.5, 89.0, 104.0, 130.0, 1000.0, 2.0 ** 24, 2.0 ** 24 + 2, 2.0 ** 25, 3e30, torch.finfo(TYPES[t]).max, math.inf]
    z = torch.cat([torch.linspace(-20, 20, 4001), torch.linspace(-0.01, 0.01, 101), torch.tensor([1e-30, 2.0 ** -126] + far),
                   -torch.tensor([1e-30, 2.0 ** -126] + far)])
    return z.to(TYPES[t])


def tail(a):
    """Q(a) to all its digits, which 1 + erf loses."""
    return torch.special.erfc(a / math.sqrt(2)) / 2


def definition(name, z):
    """The activation and its slope, with their limits at the infinities."""
    up, down = z == math.inf, z == -math.inf
    if name == "gelu":
        act = z * tail(-z)
        slope = tail(-z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        act, slope = ref.act(name, z).clone(), ref.slope(name, z).clone()
    if name != "none":
        act[up], act[down], slope[up], slope[down] = math.inf, 0.0, 1.0, 0.0
    return act, slope


def check(what, got, want, tol, z):
    assert not torch.isnan(got).any(), f"{what}: NaN at {z[torch.isnan(got)].tolist()[:8]}"
    whole = torch.isinf(want)
    assert torch.equal(got[whole], want[whole]), what
    off = (got - want).abs() - tol
    off[whole] = -1
    k = int(off.argmax())
    assert off[k] <= 0, f"{what}: {int((off > 0).sum())} off, worst at {z[k]}: {got[k]} for {want[k]}, {tol[k]:.3e} allowed"


def terms(t, z):
    """q = 1 / (1 + e^-z), 1 - q, Q(|z|), the bell over sqrt(2 pi), and what e^-z and the tail's formula are off by, relative."""
    q, r = torch.sigmoid(z), torch.sigmoid(-z)
    Q, bell = tail(z.abs()), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a = torch.nan_to_num(z.abs(), posinf=3e38).clamp_max(200.0)
    return q, r, Q, bell, a


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("name", ACTS)
def test_activations(t, name):
    z = line(t)
    M = z.numel()
    x, W = z.view(M, 1).cuda(), torch.ones(1, 1, dtype=TYPES[t], device="cuda")
    d = nf.LinearDesc(dtype=DT[t], K=1, N=1, act=ACTS.index(name))
    y = torch.empty(M, 1, dtype=TYPES[t], device="cuda")
    ws = torch.empty(max(nf.nf_linear_workspace_bytes(d, M), 1), dtype=torch.uint8, device="cuda")
    nf.nf_linear_fwd(d, M, x, W, None, None, None, y, None, ws)
    Z = z.double()
    want = definition(name, Z)[0]
    q, r, Q, _, a = terms(t, Z)
    if name == "silu":     # e^-z, the sum, the quotient, the product
        tol = torch.nan_to_num(want.abs(), posinf=0.0) * U * (r * 2 + 3 if t == "f32" else r * (2 * a + 2) + 4) + UNDER
    elif name == "gelu":   # the fit; the bell's argument and value, t, the polynomial and two products; the final sum
        fit, arg, low = (1.6e-8, 0.5, UNDER) if t == "f32" else (2.1e-6, 1.5, 4e-18)
        tol = a * Q * (fit + (14 + arg * a * a) * U) + U * torch.nan_to_num(want.abs(), posinf=0.0) + low
    else:
        tol = torch.zeros_like(Z)
    tol = tol + HALF[t] * (torch.nan_to_num(want.abs(), posinf=0.0) + tol) * (t != "f32") + TINY[t]
    check(name, y.view(-1).double().cpu(), want, tol, z)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("name", ACTS)
def test_slopes(t, name):
    """db of a single row with dy = 1 is the slope itself in fp32, whatever the type; dz is the same rounded."""
    z = line(t)
    N = z.numel()
    d = nf.LinearDesc(dtype=DT[t], K=8, N=N, act=ACTS.index(name))
    dz, db = torch.empty(1, N, dtype=TYPES[t], device="cuda"), torch.empty(N, device="cuda")
    ws = torch.empty(max(nf.nf_linear_workspace_bytes(d, 1), 1), dtype=torch.uint8, device="cuda")
    nf.nf_linear_bwd_epilogue(d, 1, torch.ones(1, N, dtype=TYPES[t], device="cuda"), z.view(1, N).cuda(), None, dz, db, ws)
    Z = z.double()
    want = definition(name, Z)[1]
    q, r, Q, bell, a = terms(t, Z)
    if name == "silu" and t == "f32":   # large and small, the larger and smaller of q and 1 - q: 3 u and 6 u
        large, small = torch.maximum(q, r), torch.minimum(q, r)
        tol = U * (10 * a * large * small + 6 * torch.where(Z < 0, small, large) + want.abs()) + UNDER
    elif name == "silu":                # q's error through q + z q (1 - q), then the two products and the sum
        dq = q * (r * (2 * a + 2) + 3) * U
        tol = (1 + a * (r - q).abs()) * dq + U * (2 * a * q * r + want.abs() + a * q * U) + UNDER
        tol = torch.where(Z >= 18, torch.full_like(tol, 2.0 ** -22), tol)   # 1 + e^-z is 1, and so is q
    elif name == "gelu":
        tol = Q * (1.6e-8 + (14 + 1.5 * a * a) * U) + a * bell * (5 + 1.5 * a * a) * U + U * (1 + want.abs()) + UNDER
    else:
        tol = torch.zeros_like(Z)
    check(name, db.double().cpu(), want, tol, z)
    check(name, dz.view(-1).double().cpu(), want, tol + HALF[t] * (want.abs() + tol) * (t != "f32") + TINY[t], z)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("name", ACTS)
def test_nan_stays(t, name):
    d = nf.LinearDesc(dtype=DT[t], K=1, N=1, act=ACTS.index(name))
    x = torch.tensor([[math.nan], [1.0]], dtype=TYPES[t], device="cuda")
    W, y = torch.ones(1, 1, dtype=TYPES[t], device="cuda"), torch.empty(2, 1, dtype=TYPES[t], device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    nf.nf_linear_fwd(d, 2, x, W, None, None, None, y, None, ws)
    assert torch.isnan(y).view(-1).tolist() == [True, False]
    if name in ("silu", "gelu"):
        dz = torch.empty(2, 1, dtype=TYPES[t], device="cuda")
        nf.nf_linear_bwd_epilogue(d, 2, torch.ones(2, 1, dtype=TYPES[t], device="cuda"), x, None, dz, None, ws)
        assert torch.isnan(dz).view(-1).tolist() == [True, False]
