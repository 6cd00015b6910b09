"""Long sums whose tests would miss a part left out, if they allowed a rounding for each term: inputs, results in 64 bits, and bounds that count the
roundings on the way of one term to its result."""
import numpy as np
import torch

from tests import layer_norm_ref, mx_ref

U = 2.0 ** -24


# ---- a layer norm's parameter gradients: sums over the rows ----

NORMS = [(300000, 9), (70000, 40), (150001, 7), (66000, 130), (40000, 520), (20000, 2048), (9000, 5000), (3000, 16400)]


def rows_deep(M, C):
    """Additions on a term's way: a thread's rows, its wave's lanes, the workgroup's waves, every 64th workgroup, and 64 lanes."""
    pieces = -(-C // 8)
    if pieces > 2048:   # parts of at least 16 rows, a thread to 8 columns
        parts = max(1, min(256, M // 16))
        return -(-M // parts) + -(-parts // 64) + 6
    if pieces <= 256:   # rows of lanes of a wave
        lanes = next(n for n in (2, 4, 8, 16, 32, 64) if n >= min(pieces, 64))
        slots, most = 256 // lanes, 1024 // (1 if pieces <= 64 else 2 if pieces <= 128 else 4)
    else:               # rows of a workgroup
        slots, most = 1, min(512 if pieces <= 512 else 256, max(64, M // 4))
    blocks = min(-(-M // slots), most)
    return -(-M // (blocks * slots)) + 6 + 4 + -(-blocks // 64) + 6


def norm_case(M, C, T):
    """x, dy, mean, rstd; dy follows the normalised rows and has a mean, so that every row moves both sums the same way."""
    g = torch.Generator().manual_seed(M + C)
    x, _, _, dy, _ = layer_norm_ref.case(g, M, C, T)
    _, mean, rstd = layer_norm_ref.forward(x.double(), 1.0, 0.0, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    dy = (0.5 * dy.double() + 0.5 * xh + 0.5).to(T)
    return x, dy, mean, rstd


def norm_sums(x, dy, mean, rstd):
    """dgamma, dbeta and what each may be off by (xh has two roundings)."""
    xh, d = (x.double() - mean.double()[:, None]) * rstd.double()[:, None], dy.double()
    deep = rows_deep(*x.shape)
    return (d * xh).sum(0), d.sum(0), 1.01 * (deep + 2) * U * (d * xh).abs().sum(0), 1.01 * deep * U * d.abs().sum(0)


# ---- products of 4-bit operands: sums along K ----

PRODUCTS = [(64, 40000, 72), (33, 65536, 64), (32, 65536, 32), (8, 30000, 40), (300, 20000, 256), (257, 8230, 300)]


def terms_deep(K):
    """Steps of fp32 (2 U, for sums that may be cut) on a term's way: 7 levels of two within an instruction of 128 terms, an instruction's sum
    to the next's, and the parts: at most 64 of them, waves of a workgroup or a split's."""
    return 14 + -(-K // 128) + 64


def four_bits(M, K, N):
    """Codes, exponent bytes and values of both operands."""
    g = torch.Generator().manual_seed(M + K + N)
    out = []
    for rows in (M, N):
        code = torch.randint(0, 16, (rows, K), generator=g).numpy().astype(np.uint8)
        byte = torch.randint(125, 130, (rows, -(-K // 32)), generator=g).numpy().astype(np.uint8)
        out.append((code, byte, torch.from_numpy(mx_ref.values(code, byte))))
    return out


def product(A, B):
    """a b^T and what it may be off by."""
    return A @ B.t(), terms_deep(A.shape[1]) * 2 * U * (A.abs() @ B.abs().t())
