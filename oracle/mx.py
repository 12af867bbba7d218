"""The microscaled 4-bit form in 64 bits, straight from its definition (numpy; test infrastructure only)."""
from __future__ import annotations

import numpy as np

BLOCK = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(X):
    """Codes (rows x padded columns) and scale bytes (rows x blocks) of float64 values, blocks along the rows.  The codes of a block
    with a NaN or an infinity are zeros here (they stand for nothing: its scale byte is 255)."""
    X = np.asarray(X, dtype=np.float64)
    rows, n = X.shape
    blocks = -(-n // BLOCK)
    x = np.zeros((rows, blocks * BLOCK))
    x[:, :n] = X
    x = x.reshape(rows, blocks, BLOCK)
    bad = ~np.isfinite(x).all(axis=2)
    x = np.where(bad[:, :, None], 0.0, x)
    amax = np.abs(x).max(axis=2, initial=0.0)
    scales = np.zeros((rows, blocks), dtype=np.int64)
    nz = amax > 0
    scales[nz] = np.clip(np.frexp(amax[nz])[1] - 1 - 2 + 127, 0, 254)
    a = np.ldexp(np.abs(x), (127 - scales)[:, :, None])          # exact in float64
    # nearest value: the distance to every one of them, ties to the even code
    d = np.abs(a[..., None] - VALUES)
    best = d.min(axis=3, keepdims=True)
    hit = d == best
    first = hit.argmax(axis=3)
    last = 7 - hit[..., ::-1].argmax(axis=3)
    codes = np.where(first % 2 == 0, first, last)
    codes = codes + 8 * np.signbit(x)
    scales[bad] = 255
    return codes.reshape(rows, -1).astype(np.uint8), scales.astype(np.uint8)


def values(codes, scales, n):
    """Values of codes and scale bytes in float64 (rows x n)."""
    rows = codes.shape[0]
    v = VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(rows, -1, BLOCK) * s[:, :, None]).reshape(rows, -1)[:, :n]


def read_back(X):
    """Q(X)."""
    X = np.asarray(X, dtype=np.float64)
    return values(*quantize(X), X.shape[1])


def bytes_of(codes):
    """Two codes a byte, the first in the lower half."""
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)


def codes_of(data):
    out = np.empty((data.shape[0], 2 * data.shape[1]), dtype=np.uint8)
    out[:, 0::2], out[:, 1::2] = data & 15, data >> 4
    return out


def product_bound(a, b, n):
    """Largest error of A B^T summed in FP32 in any order: the products are exact, and each of the n additions is off by at most
    2^-23 of the sum of magnitudes (whether it rounds or cuts)."""
    return max(n, 1) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
