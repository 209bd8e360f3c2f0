"""Pins of the dense-document oracle: hand-worked values, published vectors of the
generator, and gradients against central differences."""

import numpy as np
import pytest

from oracle import dense


def _difference(f, at, direction, step=1e-5):
    return (f(at + step * direction) - f(at - step * direction)) / (2 * step)


def test_norm_by_hand():
    x = np.array([[3.0, 4.0], [0.0, 0.0]])
    y, h = dense.rms_norm(x, np.array([2.0, 0.5]), 0.5, residual=np.array([[0.0, 0.0], [0.0, 0.0]]))
    r = np.sqrt(12.5 + 0.5)
    assert np.allclose(y, [[6 / r, 2 / r], [0, 0]], atol=0, rtol=1e-15) and np.array_equal(h, x)


@pytest.mark.parametrize("cols", [1, 2, 7])
def test_norm_gradient_against_differences(cols):
    rng = np.random.default_rng(cols)
    x, r, dy, dh = (rng.normal(size=(3, cols)) for _ in range(4))
    w, eps = rng.normal(size=cols), 0.1

    def loss(x, w):
        y, h = dense.rms_norm(x, w, eps, r)
        return (dy * y).sum() + (dh * h).sum()

    dx, dw = dense.rms_norm_backward(dy, x + r, w, eps, dh)
    for _ in range(4):
        d, e = rng.normal(size=x.shape), rng.normal(size=cols)
        # central differences: error of order step^2 and rounding / step
        assert abs(_difference(lambda v: loss(v, w), x, d) - (dx * d).sum()) < 1e-7
        assert abs(_difference(lambda v: loss(x, v), w, e) - (dw * e).sum()) < 1e-7


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_product_gradient_against_differences(act):
    rng = np.random.default_rng(11)
    x, W, b, dy = rng.normal(size=(4, 5)), rng.normal(size=(5, 3)), rng.normal(size=3), rng.normal(size=(4, 3))
    y, pre = dense.product(x, W, b, act, alpha=0.7)
    assert np.abs(pre).min() > 1e-3                     # off relu's corner
    dx, dW, db = dense.product_backward(dy, x, W, act, pre, 0.7)
    loss = lambda x, W, b: (dy * dense.product(x, W, b, act, alpha=0.7)[0]).sum()
    for _ in range(4):
        d, e, f = rng.normal(size=x.shape), rng.normal(size=W.shape), rng.normal(size=3)
        assert abs(_difference(lambda v: loss(v, W, b), x, d) - (dx * d).sum()) < 1e-7
        assert abs(_difference(lambda v: loss(x, v, b), W, e) - (dW * e).sum()) < 1e-7
        assert abs(_difference(lambda v: loss(x, W, v), b, f) - (db * f).sum()) < 1e-7


def test_activations_by_hand():
    v = np.array([-2.0, 0.0, 1.0])
    assert np.array_equal(dense.activation("relu", v), [0, 0, 1])
    assert np.allclose(dense.activation("silu", v), [-2 / (1 + np.exp(2.0)), 0, 1 / (1 + np.exp(-1.0))], rtol=1e-14)
    assert np.allclose(dense.activation("gelu", v), [-2 * 0.022750131948179212, 0, 0.8413447460685429], rtol=1e-13)
    assert np.allclose(dense.activation("gelu_tanh", v), dense.activation("gelu", v), atol=1e-3)


def test_scores_are_distances():
    # |x|^2 + (alpha = -2 product with the codebook's norms as bias) = |x - w_j|^2
    rng = np.random.default_rng(3)
    x, W = rng.normal(size=(4, 6)), rng.normal(size=(6, 9))
    y, _ = dense.product(x, W, (W ** 2).sum(0), alpha=-2.0)
    want = ((x[:, :, None] - W[None]) ** 2).sum(1)
    assert np.allclose((x ** 2).sum(1)[:, None] + y, want, rtol=1e-12)


def test_generator_published_vectors():
    # the known-answer vectors published with the generator
    assert dense.philox((0,) * 4, (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert dense.philox((0xffffffff,) * 4, (0xffffffff,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert dense.philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_dropout_keeps_the_expectation():
    x = np.ones((64, 256))
    for p in (0.0, 0.1, 0.5, 0.9):
        y = dense.dropout(x, p, seed=7, offset=3)
        # mean of 16,384 draws: five standard deviations
        assert abs(y.mean() - 1.0) <= 5 * np.sqrt(p / (1 - p) / x.size) + 1e-12
    assert not dense.dropout(x, 1.0, seed=7).any()
    r = np.full((64, 256), 2.0)
    assert np.array_equal(dense.dropout(x, 1.0, seed=7, residual=r), r)
