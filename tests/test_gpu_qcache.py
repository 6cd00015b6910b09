"""The quantised activation cache on the GPU: codes, exponents and values equal to the definition's, bit by bit."""
import numpy as np
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import pointwise_ref as ref
from tests.pointwise_ref import DT, TYPES

pytestmark = pytest.mark.gpu
FORMATS = {"int8": nf.NF_Q_INT8, "e4m3": nf.NF_Q_E4M3, "e2m1": nf.NF_Q_E2M1}


def rows(t, R, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, n, generator=g) * torch.exp(2 * torch.randn(n, generator=g))
    x[torch.rand(R, n, generator=g) < 0.3] = 0
    x[:, : min(n, 40)] = torch.round(x[:, : min(n, 40)])    # ties
    return x.to(TYPES[t])


def cache(fmt, capacity, n, labels=True):
    cb, sb = nf.nf_qcache_row_bytes(fmt, n)
    codes = torch.full((capacity + 2, cb), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((capacity + 2, sb), 0xA5, dtype=torch.uint8, device="cuda")
    return codes, scales, torch.full((capacity,), -9, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("f", FORMATS)
@pytest.mark.parametrize("R,n", [(1, 1), (3, 7), (5, 32), (4, 33), (2, 100), (3, 1000), (2, 2064), (300, 16)])
def test_rows_equal_the_definition(t, f, R, n):
    fmt = FORMATS[f]
    x = rows(t, R, n, R + n)
    codes, scales, lab = cache(fmt, R + 3, n)
    inner_c, inner_s = codes[1:-1], scales[1:-1]
    labels = torch.arange(R, dtype=torch.int32, device="cuda") * 3
    nf.nf_qcache_write(fmt, DT[t], inner_c, inner_s, lab, R + 3, n, 2, R, x.cuda(), labels)
    torch.cuda.synchronize()
    bytes_, want = ref.quantise(fmt, x.double().numpy())
    assert np.array_equal(inner_s[2:2 + R, : bytes_.shape[1]].cpu().numpy(), bytes_)
    for keep in (codes[:3], codes[3 + R:], scales[:3], scales[3 + R:]):
        assert (keep == 0xA5).all()      # other rows
    assert lab.tolist() == [-9, -9] + labels.tolist() + [-9]
    out = torch.full((R * n + 16,), -77.0, dtype=TYPES[t], device="cuda")
    lo = torch.empty(R, dtype=torch.int32, device="cuda")
    nf.nf_qcache_read(fmt, DT[t], inner_c, inner_s, lab, R + 3, n, 2, None, R, out, lo)
    assert torch.equal(out[: R * n].view(R, n).cpu(), torch.from_numpy(want).to(TYPES[t])) and torch.equal(lo, labels)
    assert (out[R * n:] == -77).all()
    idx = torch.tensor([R + 1, 2, -5, 1 << 40], dtype=torch.int64, device="cuda")   # the last two are clamped
    inner_c[0], inner_s[0], lab[0] = inner_c[2], inner_s[2], 41
    inner_c[R + 2], inner_s[R + 2], lab[R + 2] = inner_c[R + 1], inner_s[R + 1], 42
    out = torch.empty(4, n, dtype=TYPES[t], device="cuda")
    lo = torch.empty(4, dtype=torch.int32, device="cuda")
    nf.nf_qcache_read(fmt, DT[t], inner_c, inner_s, lab, R + 3, n, 0, idx, 4, out, lo)
    assert torch.equal(out.cpu(), torch.from_numpy(want[[R - 1, 0, 0, R - 1]]).to(TYPES[t]))
    assert lo.tolist() == [3 * (R - 1), 0, 41, 42]


@pytest.mark.parametrize("f", FORMATS)
def test_numbers_at_the_edges(f):
    """Zeros, subnormal and largest fp32 numbers, infinities and NaN, each in a group of its own."""
    fmt = FORMATS[f]
    top = torch.finfo(torch.float32).max
    groups = [[0.0], [-0.0, 0.0], [1e-45], [1e-40, -3e-41], [2.0 ** -126, 2.0 ** -127], [top], [-top, 1.0], [float("inf"), 1.0],
              [1.0, float("nan")], [float("-inf")], [1.0], [448.0, 1.0], [127.0, 126.5, -125.5], [6.0, 5.0, 3.5, 2.5, 0.25, 0.75],
              [464.0, 1e-3], [449.0], [127.5], [6.5, 1.0]]
    x = torch.zeros(1, 32 * len(groups))
    for i, v in enumerate(groups):
        x[0, 32 * i:32 * i + len(v)] = torch.tensor(v)
    codes, scales, lab = cache(fmt, 1, x.shape[1])
    nf.nf_qcache_write(fmt, nf.NF_F32, codes, scales, None, 1, x.shape[1], 0, 1, x.cuda(), None)
    out = torch.empty(1, x.shape[1], device="cuda")
    nf.nf_qcache_read(fmt, nf.NF_F32, codes, scales, None, 1, x.shape[1], 0, None, 1, out, None)
    bytes_, want = ref.quantise(fmt, x.double().numpy())
    assert np.array_equal(scales[0, : len(groups)].cpu().numpy(), bytes_[0])
    with np.errstate(over="ignore"):   # the largest fp32 number rounds up to an infinity, as it would in fp32
        want = want.astype(np.float32)
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("f", FORMATS)
def test_every_code_reads_as_its_number(f):
    fmt = FORMATS[f]
    book = ref.codebook(fmt)
    n = 256 if f != "e2m1" else 32
    codes = torch.zeros(1, nf.nf_qcache_row_bytes(fmt, n)[0], dtype=torch.uint8, device="cuda")
    if f == "e2m1":
        codes[0] = torch.tensor([(i % 8 * 2) | (i % 8 * 2 + 1) << 4 for i in range(16)], dtype=torch.uint8)
        want = (book + [-v for v in book]) * 2
    else:
        codes[0] = torch.arange(256)
        want = [float(i - 256 * (i > 127)) for i in range(256)] if f == "int8" else book + [float("nan")] + [-v for v in book] + [float("nan")]
    scales = torch.full((1, 16), 127 + 3, dtype=torch.uint8, device="cuda")
    out = torch.empty(1, n, device="cuda")
    nf.nf_qcache_read(fmt, nf.NF_F32, codes, scales, None, 1, n, 0, None, 1, out, None)
    assert np.array_equal(out[0].cpu().numpy(), 8 * np.array(want, np.float32), equal_nan=True)


def test_rows_past_32_bits():
    fmt, n, capacity = nf.NF_Q_INT8, 65536, 70000
    cb, sb = nf.nf_qcache_row_bytes(fmt, n)
    codes = torch.empty(capacity, cb, dtype=torch.uint8, device="cuda")
    scales = torch.empty(capacity, sb, dtype=torch.uint8, device="cuda")
    x = rows("bf16", 3, n, 8)
    nf.nf_qcache_write(fmt, nf.NF_BF16, codes, scales, None, capacity, n, capacity - 3, 3, x.cuda(), None)
    idx = torch.tensor([capacity - 1, capacity - 3], device="cuda")
    out = torch.empty(2, n, dtype=torch.bfloat16, device="cuda")
    nf.nf_qcache_read(fmt, nf.NF_BF16, codes, scales, None, capacity, n, 0, idx, 2, out, None)
    want = ref.quantise(fmt, x.double().numpy())[1]
    assert torch.equal(out.cpu(), torch.from_numpy(want[[2, 0]]).bfloat16())
