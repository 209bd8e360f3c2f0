"""fp64 oracle of the dense-document operators: the norm, the product, dropout,
and their gradients, written from the formulas in numpy."""

from __future__ import annotations

import math

import numpy as np


def rms_norm(x, weight=None, eps=0.0, residual=None):
    """(y, h): h = x + residual, y = h / sqrt(mean_c h^2 + eps) * weight."""
    h = x if residual is None else x + residual
    y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    return (y if weight is None else y * weight), h


def rms_norm_backward(dy, h, weight=None, eps=0.0, dh=None):
    """(dx, dweight) from the gradients of y and of h."""
    s = 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    g = dy if weight is None else dy * weight
    dx = s * g - h * s ** 3 * (g * h).mean(axis=1, keepdims=True)
    return (dx if dh is None else dx + dh), (dy * h * s).sum(axis=0)


# (erfc, and not 1 + erf, which loses the digits of a small share)
_below = np.vectorize(lambda v: 0.5 * math.erfc(-v / math.sqrt(2.0)), otypes=[np.float64])


def activation(name, v):
    if name == "none":
        return v
    if name == "relu":
        return np.maximum(v, 0.0)
    if name == "gelu":
        return v * _below(v)
    if name == "gelu_tanh":
        return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v * 0.5 * (1.0 + np.tanh(0.5 * v))
    raise ValueError(name)


def activation_grad(name, v):
    if name == "none":
        return np.ones_like(v)
    if name == "relu":
        return (v > 0).astype(np.float64)
    if name == "gelu":
        return _below(v) + v * np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        t = np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
        return 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * v * v)
    if name == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * v))
        return s + v * s * (1.0 - s)
    raise ValueError(name)


def product(x, W, bias=None, act="none", residual=None, alpha=1.0, x_scale=None, w_scale=None):
    """(y, pre)."""
    pre = alpha * (x @ W)
    if x_scale is not None:
        pre = pre * x_scale[:, None]
    if w_scale is not None:
        pre = pre * w_scale
    if bias is not None:
        pre = pre + bias
    y = activation(act, pre)
    return (y if residual is None else y + residual), pre


def product_backward(dy, x, W, act="none", pre=None, alpha=1.0):
    """(dx, dW, dbias)."""
    dP = dy if act == "none" else dy * activation_grad(act, pre)
    return alpha * (dP @ W.T), alpha * (x.T @ dP), dP.sum(axis=0)


def philox(counter, key, rounds=10):
    """Words of Philox4x32 (Salmon et al., SC 2011); counter of four and key of two
    Python integers below 2^32."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_bits(rows, cols, seed, offset=0):
    """The 16 random bits of every element."""
    out = np.empty((rows, (cols + 7) // 8 * 8), np.uint16)
    for r in range(rows):
        for g in range((cols + 7) // 8):
            words = philox((g, r, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
            out[r, 8 * g:8 * g + 8] = [h for w in words for h in (w & 0xFFFF, w >> 16)]
    return out[:, :cols]


def dropout(x, p, seed, offset=0, residual=None):
    t = round(65536 * p)
    keep = dropout_bits(*x.shape, seed, offset) >= t
    y = np.where(keep, x * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return y if residual is None else y + residual
