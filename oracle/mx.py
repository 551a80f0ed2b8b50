"""Microscaled 4-bit floating point in numpy, from the definition: elements, scales, the blob's bytes, and the matrix product in 64 bits.

A block of 32 columns of a row with largest magnitude a has the scale 2^s, s = max(floor(log2 a) - 2, -127); an element is the member of
0, 1/2, 1, 3/2, 2, 3, 4, 6 nearest to |x| / 2^s, ties to the member with an even mantissa bit, what is past 6 is 6.  A block that holds
an infinity or a NaN is NaN.  Plain and slow on purpose; shares no code with the library.
"""
from __future__ import annotations

import numpy as np

MEMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def encode(x):
    """x [rows, cols] -> (codes uint8 [rows, cols] of sign * 8 + member, scales uint8 [rows, blocks])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    n = -(-cols // BLOCK)
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, n), np.uint8)
    for b in range(n):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        bad = ~np.isfinite(v).all(axis=1)
        a = np.where(bad, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(axis=1))
        _, e = np.frexp(a)                                     # a = f * 2^e, f in [1/2, 1)
        s = np.where(a > 0, np.maximum(e - 1 - 2, -127), -127)
        m = np.abs(np.where(np.isfinite(v), v, 0.0)) / np.ldexp(1.0, s)[:, None]
        d = np.abs(m[:, :, None] - MEMBERS)
        near = d.min(axis=2, keepdims=True) == d               # one member, or the two around a tie
        odd = np.arange(8) % 2 == 1
        pick = np.where(near.sum(axis=2) == 2, np.argmax(near & ~odd, axis=2), np.argmax(near, axis=2))
        c = (pick + 8 * np.signbit(np.where(np.isfinite(v), v, 0.0))).astype(np.uint8)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.where(bad[:, None], 0, c)
        scales[:, b] = np.where(bad, 255, s + 127)
    return codes, scales


def decode(codes, scales):
    """The values, float64."""
    v = MEMBERS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, axis=1)[:, :codes.shape[1]]


def values(x):
    return decode(*encode(x))


def blob(codes, scales):
    """The bytes of the library's blob."""
    rows, cols = codes.shape
    n = scales.shape[1]
    nRT, nKT, pitch = -(-rows // 128), -(-cols // 128), n * 16
    off_values = 128 + nRT * nKT * 512
    total = off_values + -(-rows * pitch // 128) * 128
    out = np.zeros(total, np.uint8)
    h = out[:128].view(np.uint32)
    h[:10] = [0x584D504E, 1, rows, cols, pitch, 128, off_values & 0xFFFFFFFF, off_values >> 32, total & 0xFFFFFFFF, total >> 32]
    r, b = np.meshgrid(np.arange(rows), np.arange(n), indexing="ij")
    out[128 + ((r // 128) * nKT + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4] = scales
    words = np.zeros((rows, n * 4), np.uint32)
    for c in range(cols):
        nibble = c % 8 // 2 + 4 * (c % 2)
        words[:, c // 8] |= codes[:, c].astype(np.uint32) << np.uint32(4 * nibble)
    out[off_values:off_values + rows * pitch] = words.view(np.uint8).reshape(-1)
    return out


def linear(x, w, bias=None, residual=None, relu=False):
    """act(x w^T + bias + residual) in 64 bits; x, w the values."""
    y = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        y = y + bias
    if residual is not None:
        y = y + residual
    return np.maximum(y, 0.0) if relu else y
