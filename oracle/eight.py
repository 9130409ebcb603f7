"""Float64 definitions of the operators of towers in 8 bits and of a head with
many classes (``vfl_rmsnorm_*``, ``vfl_quantize``, ``vfl_matmul8``,
``vfl_softmax_loss_*``): test infrastructure, shares nothing with the kernels.

A matrix in 8 bits is a pair (values, power): float64 e4m3 values [rows x padded
columns] and the integer exponents [blocks x rows], standing for
values * 2^power of their block.
"""
import numpy as np

BLOCK, TOP = 128, 448.0


def e4m3_table():
    """The 256 values of e4m3 by their bits (NaN at 127 and 255)."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v[(b & 127) == 127] = np.nan
    return np.where(b & 128, -v, v)


def e4m3_round(v):
    """Magnitudes up to 448 to the nearest e4m3 value, ties to an even last bit."""
    v = np.asarray(v, np.float64)
    _, x = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(x - 1, -6) - 3)
    return np.rint(v / step) * step


def quantize(x):
    """(values, power) of a matrix: per block the smallest power of two, 2^-127 or
    more, that takes the finite magnitudes to 448 or less; NaN for what is no number."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    wide = np.zeros((rows, nb * BLOCK))
    wide[:, :cols] = x
    blocks = wide.reshape(rows, nb, BLOCK)
    fine = np.isfinite(blocks)
    top = np.where(fine, np.abs(blocks), 0.0).max(2)
    with np.errstate(divide="ignore"):
        guess = np.ceil(np.log2(top / TOP))              # may be one off
    power = np.where(top > 0, np.maximum(guess, -127), -127).astype(int)
    power += np.ldexp(TOP, power) < top
    power -= (power > -127) & (np.ldexp(TOP, power - 1) >= top)
    q = e4m3_round(np.ldexp(np.where(fine, blocks, 0.0), -power[:, :, None]))
    return np.where(fine, q, np.nan).reshape(rows, -1), power.T


def dequantize(values, power):
    return np.ldexp(values, np.repeat(power.T, BLOCK, axis=1))


def rms_stats(s, eps):
    return 1.0 / np.sqrt((s * s).sum(1) / s.shape[1] + eps)


def rms_forward(x, r, gamma, eps):
    s = x + r
    k = rms_stats(s, eps)
    return s, k, s * k[:, None] * gamma


def rms_backward(s, k, dy, ds, gamma):
    h = s * k[:, None]
    g = dy * gamma
    c = (g * h).mean(1, keepdims=True)
    return ds + k[:, None] * (g - h * c), (dy * h).sum(0)


def softmax_loss(x, w, bias, labels):
    """(loss, lse); a label outside the classes: loss 0; a class of bias -inf: out
    of the sums, loss +inf for its labels."""
    z = x @ w.T + bias
    top = z.max(1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
    has = (labels >= 0) & (labels < w.shape[0])
    at = np.where(has, labels, 0)
    zl = z[np.arange(len(z)), at]
    loss = np.where(has, np.where(np.isneginf(zl), np.inf, lse - np.where(np.isneginf(zl), 0.0, zl)), 0.0)
    return loss, lse


def softmax_grad(x, w, bias, labels, lse, dloss):
    """G = dloss (exp(z - lse) - onehot), 0 for rows without a label and classes
    taken out."""
    z = x @ w.T + bias
    p = np.exp(z - np.where(np.isneginf(lse), np.inf, lse)[:, None])
    has = (labels >= 0) & (labels < w.shape[0])
    rows = np.nonzero(has)[0]
    p[rows, labels[rows]] -= 1.0
    p[:, np.isneginf(bias)] = 0.0
    return np.where(has, dloss, 0.0)[:, None] * p
