"""Groups whose largest magnitude is a subnormal number: their exponent is the least there is, -127, and what exceeds 2^-129 has a code other
than 0.  Codes to the bit, in every call that quantises."""
import numpy as np
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import mx_ref
from tests.pointwise_ref import DT, TYPES
from tests.test_gpu_mx import check_codes, held, quantised, strides
from tests.test_gpu_pointwise import workspace

pytestmark = pytest.mark.gpu


def small(t):
    """40 rows of 96: group (r, k) has magnitudes up to a border between codes times 2^-127, or a step of the type beside it; fp16, whose subnormal
    numbers are others' normal ones, has its own."""
    T = TYPES[t]
    step = float(torch.finfo(T).tiny) * torch.finfo(T).eps   # from one subnormal number to the next
    unit = 2.0 ** -127 if t != "f16" else 2.0 ** -16
    tops = [m * unit + k * step for m in (0.125, 0.25, 0.375, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0) for k in (-1, 0, 1)]
    g = torch.Generator().manual_seed(1)
    x = torch.zeros(40, 96, dtype=torch.float64)
    for r in range(40):
        for k in range(3):
            top = tops[(3 * r + k) % len(tops)]
            # any multiples of the step below the largest, the borders among them
            v = torch.floor(top / step * torch.rand(32, generator=g, dtype=torch.float64)) * step
            v[:4] = torch.tensor([0.25, 0.75, 1.25, 1.75], dtype=torch.float64) * unit
            v = v.clamp(max=top) * torch.where(torch.rand(32, generator=g) < 0.5, -1.0, 1.0)
            v[5 + r % 20] = top
            x[r, 32 * k:32 * k + 32] = v
    assert torch.equal(x.to(T).double(), x)
    return x.to(T)


def test_the_cases_reach_the_codes():
    for t in TYPES:
        code, byte, _ = mx_ref.quantise(small(t).double().numpy())
        assert t == "f16" or (byte == 0).all() and {1, 2, 3, 9, 10, 11} <= set(code.reshape(-1).tolist())


@pytest.mark.parametrize("t", TYPES)
def test_codes(t):
    x = small(t)
    a, b = quantised(t, x)
    check_codes(a, x.double().numpy())
    check_codes(b, x.double().t().numpy())
    for rows, cols in ((True, False), (False, True)):
        p, q = quantised(t, x, rows, cols)
        check_codes(p if rows else q, (x if rows else x.t()).double().numpy())
    same = held(40, 96)
    nf.nf_qcache_write(nf.NF_Q_E2M1, DT[t], *same, None, 40, 96, 0, 40, x.cuda(), None)
    assert torch.equal(same[0], a[0]) and torch.equal(same[1], a[1])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows", [1, 8, 9, 32, 40])
def test_linear(t, rows):
    """Weights of 2^120 bring the results among ordinary numbers; sums of few small whole numbers are exact in fp32."""
    x, N = small(t)[:rows].contiguous(), 24
    up = 120 if t != "f16" else 9
    code = np.random.RandomState(rows).randint(0, 8, (N, 96)).astype(np.uint8) & np.array([2, 10], np.uint8)[np.arange(96) % 2]   # 0 and 1
    byte = np.full((N, 3), 127 + up, np.uint8)
    W = tuple(p.cuda() for p in mx_ref.pack(code, byte, strides(96)))
    d = nf.LinearDesc(dtype=DT[t], K=96, N=N, act=0)
    y, z = (torch.empty(rows, N, dtype=TYPES[t], device="cuda") for _ in range(2))
    nf.nf_mx_linear_fwd(d, rows, x.cuda(), *W, None, None, None, y, z, workspace(nf.nf_mx_linear_workspace_bytes(d, rows)))
    want = torch.from_numpy(mx_ref.quantise(x.double().numpy())[2] @ mx_ref.values(code, byte).T).to(TYPES[t])
    assert torch.equal(y.cpu(), want) and torch.equal(z.cpu(), want) and (rows == 1 or want.any())   # the first row's codes are all 0
