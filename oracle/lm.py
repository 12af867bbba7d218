"""Weights in 4 bits with a scale per group, and the cross entropy of a linear layer's outputs with its gradient, in 64 bits, straight from their
definition (numpy; test infrastructure only)."""
from __future__ import annotations

import numpy as np


def to_scale(x, kind):
    """FP32 numbers rounded to BF16 or FP16 (what overflows: the largest number), as float32."""
    x = np.asarray(x, dtype=np.float32)
    if kind == "f16":
        with np.errstate(over="ignore"):
            return np.minimum(x.astype(np.float16), np.float16(65504)).astype(np.float32)
    bits = x.view(np.uint32).astype(np.uint64)
    bits = (bits + 0x7fff + (bits >> 16 & 1)) & 0xffff0000
    return np.minimum(bits, 0x7f7f0000).astype(np.uint32).view(np.float32)


def quantize(W, group, zeros, kind):
    """Codes (p x n), scales and zero points (p x groups; 8 without) of W, whose values are FP32 numbers."""
    W = np.asarray(W, dtype=np.float32)
    p, n = W.shape
    groups = -(-n // group)
    x = np.zeros((p, groups * group), dtype=np.float32)
    x[:, :n] = W
    x = x.reshape(p, groups, group)
    bad = ~np.isfinite(x).all(axis=2)
    x = np.where(bad[:, :, None], np.float32(0), x)
    f = np.float32
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if zeros:
            lo, hi = np.minimum(x.min(axis=2), f(0)), np.maximum(x.max(axis=2), f(0))
            scale = to_scale((hi - lo) / f(15), kind)
            zero = np.where(scale > 0, np.clip(np.rint(-lo / scale), 0, 15), 0)
        else:
            scale = to_scale(np.abs(x).max(axis=2) / f(7), kind)
            zero = np.full((p, groups), 8.0)
        q = np.where(scale[:, :, None] > 0, np.clip(np.rint(x / scale[:, :, None]) + zero[:, :, None], 0, 15), zero[:, :, None])
    q = np.where(bad[:, :, None], 8.0 if not zeros else 0.0, q)
    scale = np.where(bad, np.float32(np.nan), scale)
    zero = np.where(bad, 8.0 if not zeros else 0.0, zero)
    return q.reshape(p, -1)[:, :n].astype(np.uint8), scale, zero.astype(np.uint8)


def values(codes, scales, zeros, group):
    """What codes stand for, in float64."""
    each = lambda t: np.repeat(np.asarray(t, dtype=np.float64), group, axis=1)[:, :codes.shape[1]]  # noqa: E731
    return (codes.astype(np.float64) - each(zeros)) * each(scales)


def bytes_of(codes):
    """Two codes a byte, the first in the lower half (behind the end of a row: zero)."""
    if codes.shape[1] % 2:
        codes = np.concatenate([codes, np.zeros((codes.shape[0], 1), dtype=np.uint8)], axis=1)
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)


def cross_entropy(X, W, y, ignore):
    """loss and lse per row."""
    X, W = np.asarray(X, dtype=np.float64), np.asarray(W, dtype=np.float64)
    z = X @ W.T
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    loss = np.zeros(len(y))
    for t, v in enumerate(y):
        if v != ignore:
            loss[t] = lse[t] - z[t, v] if 0 <= v < len(W) else np.nan
    return loss, lse


def slopes(X, W, y, g, ignore):
    """The gradient of the logits."""
    X, W = np.asarray(X, dtype=np.float64), np.asarray(W, dtype=np.float64)
    _, lse = cross_entropy(X, W, y, ignore)
    d = np.exp(X @ W.T - lse[:, None])
    for t, v in enumerate(y):
        if v == ignore:
            d[t] = 0
        else:
            d[t, v] -= 1
            d[t] *= g[t]
    return d


def backward(X, W, y, g, ignore):
    """dX and dW."""
    d = slopes(X, W, y, g, ignore)
    return d @ np.asarray(W, dtype=np.float64), d.T @ np.asarray(X, dtype=np.float64)
