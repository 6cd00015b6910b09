"""Matrices in 4 bits from their definition, in 64 bits on the CPU."""
import numpy as np
import torch

BOOK = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise(x):
    """Rows [R, n] (64 bits, holding fp32 numbers): codes [R, n], exponent bytes [R, groups] and the values they stand for."""
    x = np.asarray(x, np.float64)
    R, n = x.shape
    groups = -(-n // 32)
    v = np.zeros((R, groups * 32))
    v[:, :n] = x
    v = v.reshape(R, groups, 32)
    top = np.abs(v).max(2)
    bad = ~np.isfinite(top)
    E = np.full(top.shape, -127)
    for e in range(-127, 127):   # the least exponent with which the group fits
        E[(top > 6 * 2.0 ** e) & ~bad] = e + 1
    s = np.abs(np.where(bad[..., None], 0, v)) * 2.0 ** -E[..., None].astype(np.float64)
    hi = np.minimum(np.searchsorted(BOOK, s), 7)
    lo = np.maximum(hi - 1, 0)
    up, down = BOOK[hi] - s, s - BOOK[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code + 8 * np.where(bad[..., None], False, np.signbit(v))
    code = np.where(bad[..., None], 0, code)
    byte = np.where(bad, 255, E + 127).astype(np.uint8)
    return code.reshape(R, -1)[:, :n].astype(np.uint8), byte, values(code.reshape(R, -1)[:, :n], byte)


def values(code, byte):
    n = code.shape[1]
    scale = np.repeat(np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127)), 32, 1)[:, :n]
    return np.where(code >= 8, -BOOK[code % 8], BOOK[code % 8]) * scale


def pack(code, byte, strides, rest=255):
    """Rows as they lie in memory; every byte that holds nothing is ``rest``."""
    R, n = code.shape
    odd = np.pad(code, ((0, 0), (0, n % 2)))
    out, ex = np.full((R, strides[0]), rest, np.uint8), np.full((R, strides[1]), rest, np.uint8)
    out[:, : odd.shape[1] // 2] = odd[:, 0::2] | odd[:, 1::2] << 4
    if n % 2 and rest:
        out[:, n // 2] |= (rest & 15) << 4
    ex[:, : byte.shape[1]] = byte
    return torch.from_numpy(out), torch.from_numpy(ex)


def unpack(codes, n):
    q = codes.numpy()
    return np.stack([q & 15, q >> 4], -1).reshape(len(q), -1)[:, :n]
