"""Pins of the oracle of what trains and serves the dense layer: formulas against differences,
other forms of the same sums, and values that are known."""

import numpy as np

from oracle import train


def _data(M=7, N=11, K=5, seed=0):
    rng = np.random.default_rng(seed)
    labels = rng.integers(0, N, M)
    labels[2] = -1
    labels[4] = N
    return rng.normal(size=(M, K)), rng.normal(size=(K, N)), labels, rng.normal(size=N), rng.uniform(0.5, 1.5, M)


def test_cross_entropy_by_probabilities():
    x, W, labels, bias, _ = _data()
    loss, lse = train.cross_entropy(x, W, labels, bias, 0.7)
    for m in range(len(x)):
        v = [0.7 * sum(x[m, k] * W[k, n] for k in range(5)) + bias[n] for n in range(11)]
        total = sum(np.exp(v))
        assert abs(lse[m] - np.log(total)) < 1e-12
        has = 0 <= labels[m] < 11
        assert abs(loss[m] - (-np.log(np.exp(v[labels[m]]) / total) if has else 0.0)) < 1e-12


def test_cross_entropy_of_known_scores():
    # equal scores: the logarithm of the number of classes, however large the scores
    for shift in (0.0, 1e3, -1e3):
        loss, lse = train.cross_entropy(np.zeros((1, 1)), np.zeros((1, 8)), np.array([3]), np.full(8, shift))
        assert abs(loss[0] - np.log(8)) < 1e-12 and abs(lse[0] - shift - np.log(8)) < 1e-12
    bias = np.full(8, -np.inf)
    loss, lse = train.cross_entropy(np.zeros((2, 1)), np.zeros((1, 8)), np.array([3, -1]), bias)
    assert lse[0] == -np.inf and loss[0] == np.inf and loss[1] == 0.0
    bias[5] = 2.0
    loss, lse = train.cross_entropy(np.zeros((1, 1)), np.zeros((1, 8)), np.array([5]), bias)
    assert loss[0] == 0.0 and lse[0] == 2.0


def test_cross_entropy_gradient_by_differences():
    x, W, labels, bias, dloss = _data()
    dx, dW, db, g = train.cross_entropy_backward(dloss, x, W, labels, bias, -1.3)
    assert np.abs(g.sum(1)).max() < 1e-14 and not g[2].any() and not g[4].any()
    f = lambda a, b, c: (train.cross_entropy(a, b, labels, c, -1.3)[0] * dloss).sum()  # noqa: E731
    h = 1e-6
    for got, which in ((dx, 0), (dW, 1), (db, 2)):
        base = (x, W, bias)
        for at in np.ndindex(got.shape):
            up, down = [a.copy() for a in base], [a.copy() for a in base]
            up[which][at] += h
            down[which][at] -= h
            assert abs(got[at] - (f(*up) - f(*down)) / (2 * h)) < 1e-7


def test_blocks():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(130, 300))
    x[:, 128:256] = 0.0
    s = train.quantise_scale(x)
    assert s.shape == (130, 3) and (s[:, 1] == 1.0).all()
    assert np.allclose(s[5, 2] * 448, np.abs(x[5, 256:]).max())
    t = train.quantise_scale(x, 128)
    assert t.shape == (2, 3) and np.isclose(t[0, 0] * 448, np.abs(x[:128, :128]).max())
    each = train.spread(t, 130, 300, 128)
    assert each.shape == x.shape and each[127, 127] == t[0, 0] and each[128, 256] == t[1, 2]
    W = rng.normal(size=(40, 300))
    fx, fw = train.spread(s, 130, 300), train.spread(train.quantise_scale(W, 128), 40, 300, 128)
    y, pre = train.product_blocks(x / fx, fx, W / fw, fw, act="relu")
    assert np.allclose(pre, x @ W.T) and np.allclose(y, np.maximum(pre, 0))


def test_orthogonalise_moves_singular_values_alone():
    rng = np.random.default_rng(2)
    for shape in ((6, 9), (9, 6)):
        G = rng.normal(size=shape)
        u, s, v = np.linalg.svd(G, full_matrices=False)
        a, b, c = 3.4445, -4.7750, 2.0315
        s = s / np.sqrt((s * s).sum())
        for _ in range(3):
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(train.orthogonalise(G, 3, (a, b, c)), u @ np.diag(s) @ v)
    y = train.orthogonalise(G, 40, (1.5, -0.5, 0.0))
    assert np.allclose(y.T @ y, np.eye(6))
    assert not train.orthogonalise(np.zeros((3, 4)), 5, (1.5, -0.5, 0.0)).any()
