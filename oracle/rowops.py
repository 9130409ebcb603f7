"""Float64 definitions of the row operators of residual towers: dropout keyed
by Philox counters, layer norm, and the residual join of the two.

Test infrastructure only (see ``oracle/__init__.py``).

Keying of the dropout (include/vfl.h states it): the 16-bit numbers of columns
8q .. 8q+7 of global row id ``row`` are the halves (low half first) of the four
words of the Philox4x32-10 block with key = (seed mod 2**32, seed >> 32) and
counter = (step, row mod 2**32, q, 2**31 + 2**16 * (row >> 32) + tag); an
element is kept when its number is at least t = floor(65536 p + 1/2), and kept
elements are multiplied by 65536 / (65536 - t).
"""
from __future__ import annotations

import numpy as np

from .philox import MASK, philox4x32_10


def threshold(p: float) -> int:
    return int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))


def scale(p: float) -> float:
    t = threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def numbers(seed: int, step: int, tag: int, rows, n_cols: int) -> np.ndarray:
    """The 16-bit numbers of global row ids ``rows``, columns 0..n_cols-1."""
    rows = np.asarray(rows, dtype=np.uint64)[:, None]
    q = np.arange((n_cols + 7) // 8, dtype=np.uint64)[None, :]
    last = np.uint64(1 << 31) + (rows >> np.uint64(32)) * np.uint64(1 << 16) + np.uint64(tag)
    w = philox4x32_10(step & MASK, rows, q, last, seed & MASK, (seed >> 32) & MASK)
    out = np.empty((rows.shape[0], q.shape[1], 8), dtype=np.uint32)
    for i in range(4):
        out[:, :, 2 * i] = w[i] & 0xFFFF
        out[:, :, 2 * i + 1] = w[i] >> 16
    return out.reshape(rows.shape[0], q.shape[1] * 8)[:, :n_cols]


def keep_mask(p: float, seed: int, step: int, tag: int, rows, n_cols: int) -> np.ndarray:
    return numbers(seed, step, tag, rows, n_cols) >= threshold(p)


def dropout(x, p: float, keep):
    return np.where(keep, np.asarray(x, np.float64) * scale(p), 0.0)


def layer_norm(x, gamma, beta, eps: float):
    """(y, stats [rows, 2] of mean and 1 / sqrt(var + eps))."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    d = x - mean[:, None]
    k = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    return d * k[:, None] * gamma + beta, np.stack([mean, k], axis=1)


def layer_norm_backward(x, stats, gamma, dy):
    """(dx, dgamma, dbeta) for the gradient dy of y."""
    h = (np.asarray(x, np.float64) - stats[:, :1]) * stats[:, 1:]
    g = dy * gamma
    dx = stats[:, 1:] * (g - g.mean(axis=1, keepdims=True) - h * (g * h).mean(axis=1, keepdims=True))
    return dx, (dy * h).sum(axis=0), np.asarray(dy, np.float64).sum(axis=0)


def residual(x, r, p: float, keep, gamma, beta, eps: float):
    """(s, y, stats)."""
    s = r + dropout(x, p, keep)
    y, stats = layer_norm(s, gamma, beta, eps)
    return s, y, stats


def residual_backward(s, stats, gamma, dy, ds, p: float, keep):
    """(dr, dx, dgamma, dbeta) for the gradients dy of y and ds of s."""
    dr, dgamma, dbeta = layer_norm_backward(s, stats, gamma, dy)
    dr = dr + ds
    return dr, dropout(dr, p, keep), dgamma, dbeta
