"""Layer norm, 4-bit matrices and orthogonal updates: every kernel by its name in a measurement, at sizes that reach it, with its results against 64
bits.  The large references are carried out in 64 bits on the GPU."""
import numpy as np
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import mx_ref, orth_ref
from tests import pointwise_ref as ref
from tests.pointwise_ref import ACTS, DT, FUNC, HALF, SUM, TINY, TYPES
from tests.test_gpu_pointwise_records import recorded

pytestmark = pytest.mark.gpu


def held(g, rows, n):
    """Random codes and exponents, and the values they stand for (in fp32, exactly)."""
    codes, scales = nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, n)
    groups = -(-n // 32)
    code = torch.randint(0, 16, (rows, groups * 32), generator=g, dtype=torch.uint8)
    code[:, n:] = 0
    byte = torch.randint(118, 128, (rows, groups), generator=g, dtype=torch.uint8)
    q, e = torch.full((rows, codes), 0xA5, dtype=torch.uint8), torch.full((rows, scales), 0xA5, dtype=torch.uint8)
    q[:, :groups * 16] = code[:, 0::2] | code[:, 1::2] << 4
    e[:, :groups] = byte
    book = torch.tensor(np.concatenate([mx_ref.BOOK, -mx_ref.BOOK]), dtype=torch.float32)
    v = (book[code.long()].view(rows, groups, 32) * torch.exp2(byte.float() - 127)[..., None]).view(rows, -1)[:, :n].contiguous()
    return q.cuda(), e.cuda(), v.cuda()


LARGE = {"mx_product_256x256": 1}
PARTS = lambda side: {f"mx_product_{side}x{side}": 1, "mx_product_finish": 1}  # noqa: E731
PRODUCTS = [("f32", 4059, 1, 3996, LARGE), ("f32", 4059, 100, 3996, LARGE), ("f32", 3841, 260, 4096, LARGE), ("bf16", 4096, 2400, 4001, LARGE), ("f16", 4000, 2697, 4095, LARGE),
            ("f32", 16383, 385, 1020, LARGE), ("bf16", 2000, 2080, 2100, {"mx_product_128x128": 1}), ("f32", 1930, 2300, 2177, {"mx_product_128x128": 1}),
            ("bf16", 2043, 2100, 2041, PARTS(128)), ("f16", 2043, 1900, 2041, PARTS(128)), ("f32", 2043, 300, 2041, {"mx_product_128x128": 1}), ("bf16", 8100, 33, 1000, {"mx_product_128x128": 1}),
            ("bf16", 500, 33, 1000, {"mx_product_64x64": 1}), ("f16", 130, 2100, 70, PARTS(64)), ("bf16", 32, 1000, 70, {"mx_product_few_rows": 1}), ("f32", 7, 33, 1000, {"mx_product_few_rows": 1})]


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("t,M,K,N,kernels", PRODUCTS)
def test_products(act, t, M, K, N, kernels):
    g = torch.Generator().manual_seed(M + K + N)
    (a, sa, va), (b, sb, vb) = held(g, M, K), held(g, N, K)
    bias, r = torch.randn(N, generator=g).cuda(), torch.randn(M, N, generator=g).to(TYPES[t]).cuda()
    d = nf.LinearDesc(dtype=DT[t], K=K, N=N, act=ACTS.index(act))
    y = [torch.full((M * N + 128,), -77.25, dtype=TYPES[t], device="cuda") for _ in range(2)]
    ws = torch.full((max(1, nf.nf_mx_product_workspace_bytes(d, M)),), 255, dtype=torch.uint8, device="cuda")
    got = [recorded(lambda: nf.nf_mx_product(d, M, a, sa, b, sb, bias, r, o[64:], ws), w) for o, w in zip(y, (False, True))]
    assert got[0] == got[1] == kernels
    assert torch.equal(*y) and (y[0][:64] == -77.25).all() and (y[0][64 + M * N:] == -77.25).all()
    z = va.double() @ vb.double().t() + bias.double()
    err = (K + 2) * SUM * (va.abs().double() @ vb.abs().double().t() + bias.abs().double())
    if act != "none":
        err = 1.13 * err + FUNC * z.abs()
        z = 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    want = z + r.double()
    off = (y[0][64:64 + M * N].view(M, N).double() - want).abs()
    assert (off <= err + (HALF[t] + 2 * SUM) * (want.abs() + err) + SUM * z.abs() + TINY[t]).all(), off.max()


@pytest.mark.parametrize("rows,cols,kernel", [(True, False, "mx_quantise_rows"), (False, True, "mx_quantise_columns"), (True, True, "mx_quantise_both")])
def test_quantisation(rows, cols, kernel):
    x = torch.randn(300, 200, generator=torch.Generator().manual_seed(0)).bfloat16()
    pairs = [tuple(torch.zeros(r, n, dtype=torch.uint8, device="cuda") for n in nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, c)) for r, c in ((300, 200), (200, 300))]
    call = lambda: nf.nf_mx_quantise(nf.NF_BF16, 300, 200, x.cuda(), *(pairs[0] if rows else (None, None)), *(pairs[1] if cols else (None, None)))  # noqa: E731
    assert recorded(call, False) == recorded(call, True) == {kernel: 1}
    for pair, on, m in zip(pairs, (rows, cols), (x, x.t())):
        if on:
            code, byte, _ = mx_ref.quantise(m.double().numpy())
            assert np.array_equal(mx_ref.unpack(pair[0].cpu(), m.shape[1]), code) and np.array_equal(pair[1][:, :byte.shape[1]].cpu().numpy(), byte)


@pytest.mark.parametrize("M,kernels", [(32, {"mx_linear_few_rows": 1}), (33, {"mx_quantise_rows": 1, "mx_product_64x64": 1}), (300, {"mx_quantise_rows": 1, "mx_product_64x64": 1})])
def test_linear(M, kernels):
    x, (W, e, _) = torch.randn(M, 130).half().cuda(), held(torch.Generator().manual_seed(0), 50, 130)
    d = nf.LinearDesc(dtype=nf.NF_F16, K=130, N=50, act=0)
    y, ws = torch.empty(M, 50, dtype=torch.float16, device="cuda"), torch.empty(max(1, nf.nf_mx_linear_workspace_bytes(d, M)), dtype=torch.uint8, device="cuda")
    assert recorded(lambda: nf.nf_mx_linear_fwd(d, M, x, W, e, None, None, None, y, None, ws), False) == kernels


def orth_kernels(sym, app, parts=False, steps=2):
    got = {"orth_squares": 1, "orth_start": 1, f"orth_gram_{sym}x{sym}": steps, f"orth_poly_{sym}x{sym}": steps, f"orth_last_{app}x{app}": 1}
    if steps > 1:
        got[f"orth_apply_{app}x{app}"] = steps - 1
    return {**got, "orth_parts": steps} if parts else got


def on_gpu(g, steps, eps):
    x = g / (g.square().sum().sqrt() + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for a, b, c in steps:
        a, b, c = (float(np.float32(v)) for v in (a, b, c))
        A = x @ x.t().contiguous()
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.t() if tall else x


ORTH = [([(16, 27)], {"orth_small_4_waves": 1}), ([(64, 64)], {"orth_small_16_waves": 1}), ([(64, 200), (512, 10)], {"orth_small_16_waves": 1}), ([(64, 576)], orth_kernels(64, 64)),
        ([(1000, 1000)], orth_kernels(64, 64)), ([(500, 2050)], orth_kernels(64, 64, True)), ([(1700, 1690)], orth_kernels(96, 128)), ([(2040, 2048)], orth_kernels(96, 128)), ([(2300, 2301)], orth_kernels(128, 128)),
        ([(9000, 700)], orth_kernels(64, 128, True)), ([(1000, 1500), (1400, 1300), (700, 4000)], orth_kernels(64, 128, True))]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("shapes,kernels", ORTH)
def test_orthogonal_updates(t, shapes, kernels):
    gen, steps = torch.Generator().manual_seed(len(shapes)), orth_ref.MUON[:2]
    g = [orth_ref.gradient(gen, *s).to(TYPES[t]).cuda() for s in shapes]
    y = [[torch.full((s[0] * s[1] + 128,), -77.25, dtype=TYPES[t], device="cuda") for s in shapes] for _ in range(2)]
    d = nf.orth_desc(steps, 1e-7)
    ws = torch.full((nf.nf_orthogonalise_workspace_bytes(d, shapes),), 255, dtype=torch.uint8, device="cuda")
    for o, as_run in zip(y, (False, True)):
        outs = [v[64:64 + s[0] * s[1]].view(s) for v, s in zip(o, shapes)]
        assert recorded(lambda: nf.nf_orthogonalise(d, DT[t], g, outs, ws), as_run) == kernels
    for k, s in enumerate(shapes):
        assert torch.equal(y[0][k], y[1][k])
        assert (y[0][k][:64] == -77.25).all() and (y[0][k][64 + s[0] * s[1]:] == -77.25).all()
        want = on_gpu(g[k].double(), steps, 1e-7)
        off = (on_gpu(g[k].float(), steps, 1e-7).double() - want).norm()   # the steps' own amplification of roundings; ours are at 2^-22 for 2^-24, both doubled
        got = y[0][k][64:64 + s[0] * s[1]].view(s).double()
        assert (got - want).norm() <= (8 * off + 2.0 ** -20 * want.norm()) * (1 + HALF[t]) + HALF[t] * want.norm() + TINY[t] * got.numel() ** 0.5


@pytest.mark.parametrize("C,forward,backward", [(96, "layernorm_fwd", "layernorm_bwd"), (16384, "layernorm_fwd", "layernorm_bwd"), (16392, "layernorm_fwd_long", "layernorm_bwd_long")])
def test_layer_norm(C, forward, backward):
    M = 40
    x, dy = torch.randn(M, C).bfloat16().cuda(), torch.randn(M, C).bfloat16().cuda()
    d = nf.LayerNormDesc(dtype=nf.NF_BF16, C=C, eps=1e-5)
    y, mean, rstd, dg, db = torch.empty_like(x), *(torch.empty(n, device="cuda") for n in (M, M, C, C))
    ws = torch.empty(nf.nf_layernorm_workspace_bytes(d, M), dtype=torch.uint8, device="cuda")
    assert recorded(lambda: nf.nf_layernorm_fwd(d, M, x, None, None, y, mean, rstd), False) == {forward: 1}
    names = recorded(lambda: nf.nf_layernorm_bwd(d, M, dy, x, None, mean, rstd, None, y, dg, db, ws), False)
    assert set(names) == ({backward, "layernorm_sums"} if C <= 16384 else {backward, "layernorm_columns", "layernorm_sums"}), names
