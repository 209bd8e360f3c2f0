"""fp64 oracle of what the dense layer is trained by and served with: cross entropy and
its gradients, blocks of 8 bits and their product, orthogonalised updates, written from
the formulas in numpy."""

from __future__ import annotations

import numpy as np

from .dense import activation

BLOCK = 128


def scores(x, W, bias=None, alpha=1.0):
    v = alpha * (x @ W)
    return v if bias is None else v + bias


def cross_entropy(x, W, labels, bias=None, alpha=1.0):
    """(loss, lse)."""
    v = scores(x, W, bias, alpha)
    N = v.shape[1]
    with np.errstate(divide="ignore", invalid="ignore"):
        top = v.max(axis=1)
        base = np.where(np.isneginf(top), 0.0, top)
        lse = base + np.log(np.exp(v - base[:, None]).sum(axis=1))
        has = (labels >= 0) & (labels < N)
        own = v[np.arange(len(v)), np.where(has, labels, 0)]
        loss = np.where(has, np.where(np.isneginf(lse), np.inf, lse - own), 0.0)
    return loss, lse


def cross_entropy_backward(dloss, x, W, labels, bias=None, alpha=1.0):
    """(dx, dW, dbias, g)."""
    v = scores(x, W, bias, alpha)
    M, N = v.shape
    _, lse = cross_entropy(x, W, labels, bias, alpha)
    has = (labels >= 0) & (labels < N) & ~np.isneginf(lse) & (dloss != 0)
    with np.errstate(invalid="ignore"):
        g = np.exp(v - lse[:, None])
    g[np.arange(M)[has], labels[has]] -= 1.0
    g = np.where(has[:, None], g * dloss[:, None], 0.0)
    return alpha * (g @ W.T), alpha * (np.where(has[:, None], x, 0.0).T @ g), g.sum(axis=0), g


def quantise_scale(x, block_rows=1):
    """The factors of x's blocks."""
    rows, cols = x.shape
    R, KB = -(-rows // block_rows), -(-cols // BLOCK)
    a = np.zeros((R * block_rows, KB * BLOCK))
    a[:rows, :cols] = np.abs(x)
    top = a.reshape(R, block_rows, KB, BLOCK).max(axis=(1, 3))
    return np.where(top == 0, 1.0, np.maximum(top / 448.0, 2.0 ** -126))


def spread(scale, rows, cols, block_rows=1):
    """Each element's factor."""
    return np.repeat(np.repeat(scale, block_rows, axis=0)[:rows], BLOCK, axis=1)[:, :cols]


def product_blocks(x, x_scale, W, w_scale, bias=None, act="none", residual=None, alpha=1.0):
    """(y, pre): x [M, K] and W [N, K] as codes' values, with each element's factor."""
    pre = alpha * ((x * x_scale) @ (W * w_scale).T)
    if bias is not None:
        pre = pre + bias
    y = activation(act, pre)
    return (y if residual is None else y + residual), pre


def orthogonalise(G, steps, coefficients):
    n = np.sqrt((G * G).sum())
    X = G / n if n else G
    if G.shape[0] > G.shape[1]:
        X = X.T
    a, b, c = coefficients
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if G.shape[0] > G.shape[1] else X
