"""Every kernel of the linear layer, named by the measurement's records, against 64 bits: tiles of 256, 128 and 64, whole and in parts,
rows of whole 16 bytes and odd ones, with rows, columns and terms that end inside a tile or a step, and sums shorter than the
stages that the tiles of 256 keep in flight."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import pointwise_ref as ref
from tests.pointwise_ref import ACTS, DT, FUNC, HALF, SUM, TINY, TYPES
from tests.test_gpu_pointwise import Out, workspace

pytestmark = pytest.mark.gpu
# an activation's own error relative to |z|: fp32 counts some eight roundings, 16 bits the short forms'
ACT = {"f32": 8 * SUM, "bf16": FUNC, "f16": FUNC}


def randn(g, *shape, T, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(T)


def recorded(call, as_run=True):
    nf.nf_prof_begin_as_run() if as_run else nf.nf_prof_begin()
    try:
        call()
    finally:
        got = nf.nf_prof_end()
    return {r["kernel"] for r in got}


def close(name, out, want, tol):
    torch.cuda.synchronize()
    assert (out.all[:out.band] == -77.25).all() and (out.all[out.band + out.n:] == -77.25).all(), f"{name}: written outside"
    got = out.t.double()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    off = (got - want).abs() - tol
    worst = int(off.argmax())
    assert off.max() <= 0, f"{name}: {int((off > 0).sum())} of {off.numel()} off, worst {got.reshape(-1)[worst]} for {want.reshape(-1)[worst]}"


def forward(t, M, K, N, names, act="gelu", p=0.1, res=True, z=True):
    g = torch.Generator(device="cuda").manual_seed(M * 31 + K * 7 + N)
    T = TYPES[t]
    x, W, b = randn(g, M, K, T=T), randn(g, N, K, T=T, scale=K ** -0.5), randn(g, N, T=torch.float32, scale=0.1)
    r = randn(g, M, N, T=T) if res else None
    drop = nf.DropoutDesc(p, 0x123456789ABCDEF0, 5) if p else None
    d = nf.LinearDesc(dtype=DT[t], K=K, N=N, act=ACTS.index(act))
    ws = workspace(nf.nf_linear_fwd_workspace_bytes(d, M))
    y, zz = Out(M, N, dtype=T), Out(M, N, dtype=T) if z else None
    got = recorded(lambda: nf.nf_linear_fwd(d, M, x, W, b, r, drop, y.t, zz.t if z else None, ws))
    assert got == set(names), got
    X, w, B = x.double(), W.double(), b.double()
    Z = X @ w.t() + B
    err = (K + 2) * SUM * (X.abs() @ w.abs().t() + B.abs())
    if z:
        close("z", zz, Z, err + HALF[t] * Z.abs() + TINY[t])
    keep = ref.keep_scale(M, N, p, 0x123456789ABCDEF0, 5).cuda()
    v = ref.act(act, Z) * keep
    tol = (1.13 * err + ACT[t] * Z.abs()) * keep
    Y = v + r.double() if res else v
    close("y", y, Y, tol + (HALF[t] + 2 * SUM) * (Y.abs() + tol) + SUM * v.abs() + TINY[t])


WIDE = [(60101, 200, 200), (28901, 264, 456), (14401, 1000, 1000)]


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("M,K,N", WIDE)
def test_forward_in_tiles_of_256(t, M, K, N):
    forward(t, M, K, N, ["linear_fwd_256x256"])


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_forward_in_tiles_of_256_without_its_epilogue(t):
    forward(t, 60101, 200, 200, ["linear_fwd_256x256"], act="none", p=0.0, res=False, z=False)
    forward(t, 60101, 200, 200, ["linear_fwd_256x256"], act="relu", p=0.0, res=True, z=False)
    forward(t, 60101, 200, 200, ["linear_fwd_256x256"], act="silu", p=0.25, res=False, z=True)


BOTH = ("bf16", "f16")
TILES = [(BOTH, 1803, 728, 1744, "128x128", False), (BOTH, 936, 2824, 1128, "128x128", True), (("f32",), 2451, 1192, 1240, "128x128", False),
         (("f32",), 1899, 1860, 1385, "128x128", True), (BOTH, 2576, 231, 2408, "128x128_odd", False), (BOTH, 1619, 2119, 620, "128x128_odd", True),
         (("f32",), 2763, 82, 2573, "128x128_odd", False), (("f32",), 1326, 859, 1577, "128x128_odd", True), (TYPES, 4200, 72, 100, "64x64", False),
         (BOTH, 4200, 75, 99, "64x64_odd", False), (("f32",), 4200, 75, 99, "64x64_odd", False), (BOTH, 99, 1056, 72, "64x64", True),
         (BOTH, 99, 1085, 75, "64x64_odd", True), (("f32",), 99, 556, 72, "64x64", True), (("f32",), 99, 555, 75, "64x64_odd", True)]
TILES = [(t, *c[1:]) for c in TILES for t in c[0]]


@pytest.mark.parametrize("t,M,K,N,name,parts", TILES)
def test_forward_in_tiles(t, M, K, N, name, parts):
    names = ["linear_fwd_" + name] + ["linear_fwd_finish"] * parts
    forward(t, M, K, N, names)
    forward(t, M, K, N, names, act="silu", p=0.0, res=False, z=False)


FEW = [("", {"f32": 40, "bf16": 40, "f16": 72}), ("_odd", {"f32": 37, "bf16": 39, "f16": 45}), ("_long", {"f32": 516, "bf16": 1032, "f16": 520}),
       ("_long_odd", {"f32": 513, "bf16": 1021, "f16": 519})]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,rows", [(1, 8), (7, 8), (13, 16), (29, 32), (50, 64), (64, 64)])
@pytest.mark.parametrize("form,K", FEW)
def test_forward_of_few_rows(t, M, rows, form, K):
    k = K[t] if t != "f32" or M <= 32 or K[t] <= 512 else K[t] - 216   # more than 32 rows come here with sums of up to 2 KB
    k = k if M <= 32 or k < 1000 else k - 400
    forward(t, M, k, 45, [f"linear_fwd_{rows}_rows{form}"])
    forward(t, M, k, 45, [f"linear_fwd_{rows}_rows{form}"], act="relu", p=0.0, res=False, z=False)


# shape, dx's tiles, dW's, "odd" rows, parts of dx and of dW
GRADIENTS = [
    (BOTH, 50001, 200, 8, 256, 64, False, False, True), (BOTH, 50001, 200, 40, 256, 64, False, False, True), (BOTH, 50001, 200, 264, 256, 64, False, False, True),
    (BOTH, 34, 3496, 4008, 64, 256, False, None, False), (BOTH, 201, 3496, 4008, None, 256, False, None, False), (BOTH, 2213, 3864, 2168, 256, 256, False, False, False),
    (BOTH, 2935, 1368, 712, 128, 128, False, False, True), (BOTH, 1127, 944, 2864, 128, None, False, True, None), (BOTH, 1732, 1784, 736, 128, 64, False, False, False),
    (BOTH, 721, 1712, 1848, 64, 128, False, False, False), (BOTH, 1676, 1207, 1827, 128, 128, True, True, True), (BOTH, 2066, 2978, 206, 128, None, True, False, None),
    (BOTH, 195, 1764, 3520, None, 128, True, None, False), (BOTH, 920, 1130, 2173, 128, 64, True, True, False), (BOTH, 2197, 791, 1236, 64, 128, True, False, True),
    (("f32",), 1271, 2680, 1236, 128, 128, False, False, False), (("f32",), 1302, 2388, 1196, 128, 64, False, False, False), (("f32",), 1290, 1648, 1924, 64, 128, False, True, False),
    (("f32",), 1724, 856, 2920, None, 128, False, None, True), (("f32",), 2059, 1272, 1988, 128, None, False, True, None), (("f32",), 858, 1282, 1706, 128, 128, True, True, True),
    (("f32",), 785, 1419, 1316, 128, 64, True, True, False), (("f32",), 1338, 705, 1562, 64, 128, True, True, True), (("f32",), 1675, 3613, 292, 128, None, True, False, None),
    (("f32",), 67, 3154, 2269, None, 128, True, None, False), (TYPES, 161, 72, 200, 64, 64, False, None, None), (TYPES, 161, 71, 201, 64, 64, True, None, None)]
GRADIENTS = [(t, *c[1:]) for c in GRADIENTS for t in c[0]]


@pytest.mark.parametrize("t,M,K,N,bx,bw,odd,px,pw", GRADIENTS)
def test_gradients(t, M, K, N, bx, bw, odd, px, pw):
    g = torch.Generator(device="cuda").manual_seed(M + 3 * K + 5 * N)
    T = TYPES[t]
    dz, x, W = randn(g, M, N, T=T, scale=N ** -0.5), randn(g, M, K, T=T), randn(g, N, K, T=T)
    d = nf.LinearDesc(dtype=DT[t], K=K, N=N, act=0)
    ws = workspace(nf.nf_linear_workspace_bytes(d, M))
    dx, dW, dx2, dW2 = Out(M, K, dtype=T), Out(N, K), Out(M, K, dtype=T), Out(N, K)
    apart = recorded(lambda: nf.nf_linear_bwd(d, M, dz, x, W, dx.t, dW.t, ws), as_run=False)
    as_run = recorded(lambda: nf.nf_linear_bwd(d, M, dz, x, W, dx2.t, dW2.t, ws))
    tail = "_odd" if odd else ""
    for which, b, parts in (("dx", bx, px), ("dw", bw, pw)):
        assert b is None or f"linear_{which}_{b}x{b}{tail}" in apart, apart
        assert parts is None or (f"linear_{which}_finish" in apart) == parts, apart
    if 256 not in (bx, bw) and None not in (bx, bw):
        assert f"linear_gradients_{bx}_{bw}{tail}" in as_run, as_run
    D, X, w = dz.double(), x.double(), W.double()
    want = D @ w
    close("dx", dx, want, (N + 2) * SUM * (D.abs() @ w.abs()) + HALF[t] * want.abs() + TINY[t])
    want = D.t() @ X
    close("dW", dW, want, (M + 2) * SUM * (D.abs().t() @ X.abs()))
    assert torch.equal(dx2.t, dx.t) and torch.equal(dW2.t, dW.t)


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_infinities_stay_in_their_rows_and_columns(t):
    """A row of x with an infinity and a NaN in W, in the last terms of tiles of 256: their products only."""
    M, K, N = 60101, 200, 200
    T = TYPES[t]
    x, W = torch.ones(M, K, dtype=T, device="cuda"), torch.ones(N, K, dtype=T, device="cuda")
    x[60100, 199], x[255, 0], W[199, 199] = float("inf"), float("-inf"), float("nan")
    d = nf.LinearDesc(dtype=DT[t], K=K, N=N, act=0)
    y = torch.empty(M, N, dtype=T, device="cuda")
    assert recorded(lambda: nf.nf_linear_fwd(d, M, x, W, None, None, None, y, None, None)) == {"linear_fwd_256x256"}
    want = torch.full((M, N), 200.0, device="cuda")
    want[60100], want[255], want[:, 199] = float("inf"), float("-inf"), float("nan")
    assert torch.equal(y.float().nan_to_num(9.0, 1e9, -1e9), want.nan_to_num(9.0, 1e9, -1e9))


@pytest.mark.parametrize("M,K,N,name", [(60101, 200, 200, "256x256"), (60101, 192, 200, "128x128"), (60101, 200, 184, "64x64"), (20000, 256, 512, "64x64"),
                                        (33770, 512, 136, "64x64"), (40000, 1024, 1000, "128x128"), (65536, 512, 512, "256x256")])
def test_both_sides_of_the_forward_rule_for_256(M, K, N, name):
    """Empty quarters of tiles, short sums and rounds that are not nearly whole go to smaller tiles."""
    x, W = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(N, K, dtype=torch.bfloat16, device="cuda")
    x[:, 3], W[:, 3] = 2, 3
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    d = nf.LinearDesc(dtype=nf.NF_BF16, K=K, N=N, act=0)
    ws = workspace(nf.nf_linear_fwd_workspace_bytes(d, M))
    assert recorded(lambda: nf.nf_linear_fwd(d, M, x, W, None, None, None, y, None, ws)) == {"linear_fwd_" + name}
    assert (y == 6).all()


def test_every_kernel_is_among_these_cases():
    """The tables above name all tile kernels; their tests assert that the calls took them."""
    fwd = {"linear_fwd_" + c[4] for c in TILES} | {"linear_fwd_256x256"}
    assert fwd == {f"linear_fwd_{b}x{b}{o}" for b in (64, 128) for o in ("", "_odd")} | {"linear_fwd_256x256"}
    for t in TYPES:
        rows = [c for c in GRADIENTS if c[0] == t]
        tiles = {64, 128} | ({256} if t != "f32" else set())
        for k in (4, 5):
            assert {(c[k], c[6]) for c in rows if c[k]} == {(b, o) for b in tiles for o in (False, True)} - {(256, True)}
        assert {(c[4], c[5], c[6]) for c in rows if 256 not in c[4:6] and None not in c[4:6]} == {(a, b, o) for a in (64, 128) for b in (64, 128) for o in (False, True)}
