"""The operators around the products of a block, in fp64: dropout masks, activations, epilogues and layer norm, with their gradients.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  The definitions are those of include/metis.h.
"""
import numpy as np
from scipy.special import erfc, expit

from oracle import rng

MASK_TAG = 16


def mask(p, seed, step, rows, cols):
    """Factors [len(rows), cols] of the elements of the given rows."""
    t = int(np.floor(65536 * p + 0.5))
    rows = np.asarray(rows, dtype=np.uint64)
    blocks = np.arange((cols + 7) // 8, dtype=np.uint64)
    shape = (len(rows), len(blocks))
    c = np.stack([np.broadcast_to(blocks[None, :], shape), np.broadcast_to(rows[:, None], shape), np.full(shape, MASK_TAG, np.uint64),
                  np.full(shape, step % (1 << 32), np.uint64)], -1)
    w = rng.philox4x32_10(c, np.array([seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF], dtype=np.uint64)).astype(np.int64)
    h = np.stack([w & 0xFFFF, w >> 16], -1).reshape(len(rows), -1)[:, :cols]
    return np.where(h >= t, 65536.0 / (65536 - t), 0.0)


_C = np.sqrt(2 / np.pi)


def _inner(z):
    return 2 * _C * (z + 0.044715 * z ** 3)


def act(name, z):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "gelu":
        return 0.5 * z * erfc(-z / np.sqrt(2))
    if name == "gelu_tanh":
        return z * expit(_inner(z))
    if name == "silu":
        return z * expit(z)
    return z


def slope_terms(name, z):
    """The two terms whose sum is the activation's derivative (their magnitudes set how far it may be off)."""
    if name == "relu":
        return np.where(z > 0, 1.0, 0.0), np.zeros_like(z)
    if name == "gelu":
        return 0.5 * erfc(-z / np.sqrt(2)), z * np.exp(-0.5 * z * z) * 0.5 * _C
    if name == "gelu_tanh":
        x = _inner(z)
        return expit(x), z * expit(x) * expit(-x) * 2 * _C * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        return expit(z), z * expit(z) * expit(-z)
    return np.ones_like(z), np.zeros_like(z)


def layernorm(x, weight, bias, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mean) * rstd
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, np.concatenate((mean, rstd), 1)


def layernorm_grads(dy, x, stats, weight, add):
    mean, rstd = stats[:, :1], stats[:, 1:]
    xh = (x - mean) * rstd
    g = dy if weight is None else dy * weight
    dx = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    if add is not None:
        dx = dx + add
    return dx, (dy * xh).sum(0), dy.sum(0)
