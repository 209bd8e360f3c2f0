"""Cross entropy and its gradients on the GPU against the fp64 oracle.

Tolerances (u = 2^-24, t = half a unit of x's type):
  a score, a sum of K fp32 products, is within 2 K u of the sum of their magnitudes (the matrix
  cores add them) and u of itself and of its bias: dv;
  lse is within the largest dv of its document, the exponentials' and the logarithm's 2^-18 (a
  power of two whose argument is off by |v - max| u, weighted by itself, and units of
  fp32), the sum's depth (N / 16 + 64) u, and 2 u of itself;
  a probability is within dv + dlse + 2^-18 of itself; g adds t of itself where it is rounded for
  the products, the products 2 n u of the magnitudes, each output its own t."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from dense_plan import CLASSES  # noqa: E402
from oracle import train as oracle  # noqa: E402

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"
T = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f16": 2.0 ** -24, "bf16": 2.0 ** -126}
U = 2.0 ** -24


def _np(t):
    return t.double().cpu().numpy()


def _view(values, dtype, pad, fill=float("nan")):
    """values as a view into a wider array whose other columns hold `fill`."""
    rows, cols = values.shape
    wide = torch.full((rows, cols + pad), fill, dtype=torch.float32, device=DEV).to(dtype)
    wide[:, :cols] = torch.as_tensor(values, dtype=torch.float32, device=DEV).to(dtype)
    return wide[:, :cols]


def _near(got, want, tol, what):
    got = _np(got)
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4],
                           np.broadcast_to(tol, want.shape)[bad][:4])


def _inputs(M, N, K, kind, layout, pad=0, seed=0, spread=1.0, ignored=0.2):
    rng = np.random.default_rng(seed + M * 31 + N * 7 + K)
    x = _view(rng.normal(size=(M, K)), T[kind], pad)
    W = rng.normal(size=(N, K)) * spread * K ** -0.5
    W = _view(W, T[kind], pad).t() if layout == "unit" else _view(W.T, T[kind], pad)
    labels = rng.integers(0, N, M)
    labels[rng.random(M) < ignored] = -1
    if M > 4:
        labels[1], labels[2] = N, 2 ** 31 - 1              # no classes either
    bias = torch.as_tensor(rng.normal(size=N) * 0.3, dtype=torch.float32, device=DEV)
    dloss = torch.as_tensor(rng.uniform(0.5, 1.5, M) / M, dtype=torch.float32, device=DEV)
    return x, W, torch.as_tensor(labels, dtype=torch.int32, device=DEV), bias, dloss


def _dv(x, W, v, bias, alpha):
    K = x.shape[1]
    return np.abs(alpha) * 2 * K * U * (np.abs(x) @ np.abs(W)) + 2 * U * (np.abs(v) + (0 if bias is None else np.abs(bias)))


def _check(x, W, labels, bias, dloss, alpha, kind):
    xn, Wn, ln, bn = _np(x), _np(W), labels.cpu().numpy().astype(np.int64), None if bias is None else _np(bias)
    loss, lse = som.som_cross_entropy(x, W, labels, bias, alpha)
    want, want_lse = oracle.cross_entropy(xn, Wn, ln, bn, alpha)
    v = oracle.scores(xn, Wn, bn, alpha)
    N, K = v.shape[1], xn.shape[1]
    dv = _dv(xn, Wn, v, bn, alpha)
    dlse = dv.max(1) + 2.0 ** -18 + (N / 16 + 64) * U + 2 * U * np.abs(want_lse)
    _near(lse, want_lse, dlse, "lse")
    has = (ln >= 0) & (ln < N)
    own = np.where(has, dv[np.arange(len(v)), np.where(has, ln, 0)], 0.0)
    _near(loss, want, has * (dlse + own + 2 * U * np.abs(want)), "loss")

    dx, dW, dbias = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias, alpha)
    wx, wW, wb, g = oracle.cross_entropy_backward(_np(dloss), xn, Wn, ln, bn, alpha)
    assert dx.dtype == x.dtype and dW.dtype == x.dtype and dbias.dtype == torch.float32 and dW.stride(0) == (1 if W.stride(0) == 1 and W.shape[0] > 1 else dW.stride(0))
    d = _np(dloss)[:, None]
    p = np.where(has[:, None], np.exp(v - want_lse[:, None]), 0.0) * np.abs(d)
    dg = p * (np.expm1(dv + dlse[:, None]) + 2.0 ** -18) + 4 * U * np.abs(g)
    M = len(v)
    _near(dbias, wb, dg.sum(0) + (M + 8) * U * np.abs(g).sum(0), "dbias")
    # rounded for the products: the smallest fp16 step of g scaled so that max |dloss| is 2^14 at least
    dg = dg + HALF[kind] * np.abs(g) + (2.0 ** -25 * np.abs(d).max() / 2.0 ** 13 if kind == "f16" else 0.0)
    ax, aW = np.abs(xn), np.abs(Wn)
    _near(dx, wx, abs(alpha) * (dg @ aW.T + 2 * N * U * (np.abs(g) @ aW.T)) * (1 + HALF[kind]) + HALF[kind] * np.abs(wx)
          + TINY[kind] + 4 * U * np.abs(wx), "dx")
    _near(dW, wW, abs(alpha) * (ax.T @ dg + 2 * M * U * (ax.T @ np.abs(g))) * (1 + HALF[kind]) + HALF[kind] * np.abs(wW)
          + TINY[kind] + 4 * U * np.abs(wW), "dW")
    assert not dx[~torch.as_tensor(has, device=DEV)].any()
    return loss, lse, dx, dW, dbias


SHAPES = [(1, 1, 1), (1, 2, 5), (2, 1, 64), (3, 7, 1), (4, 300, 64), (5, 1000, 72), (17, 129, 200), (33, 257, 129),
          (64, 1024, 512), (100, 777, 65), (130, 4097, 63), (257, 255, 1030), (300, 3001, 96), (515, 2051, 40),
          (1001, 777, 500), (2, 9000, 33), (1, 5000, 2100), (20, 520, 6000)]


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_loss_and_gradients(M, N, K, layout, kind):
    x, W, labels, bias, dloss = _inputs(M, N, K, kind, layout, pad=(M + N) % 3 * 4)
    _check(x, W, labels, bias, dloss, 1.0, kind)


@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("alpha,spread,with_bias", [(-2.0, 1.0, True), (0.05, 8.0, False), (1.0, 12.0, True), (0.0, 1.0, True)])
def test_scales_and_wide_scores(alpha, spread, with_bias, layout):
    x, W, labels, bias, dloss = _inputs(200, 600, 256, "bf16", layout, spread=spread)
    _check(x, W, labels, bias if with_bias else None, dloss, alpha, "bf16")


def test_large_tiles():
    # 256 x 256 and 256 x 128 tiles, columns and rows that end inside them
    for M, N, K in ((1000, 20001, 64), (2049, 6000, 128), (4100, 2056, 64)):
        x, W, labels, bias, dloss = _inputs(M, N, K, "f16", "unit" if N % 2 else "feature")
        _check(x, W, labels, bias, dloss, 0.7, "f16")


def _double(x, W, labels, bias, alpha, dloss):
    """The definition in 64 bits on the device."""
    X, V = x.double(), W.double().contiguous()
    v = alpha * torch.mm(X, V) + bias.double()
    lse = torch.logsumexp(v, 1)
    has = (labels >= 0) & (labels < W.shape[1])
    rows = torch.arange(len(v), device=DEV)
    own = v[rows, labels.clamp(0, W.shape[1] - 1).long()]
    g = torch.exp(v - lse[:, None])
    g[rows[has], labels[has].long()] -= 1.0
    g *= (dloss.double() * has)[:, None]
    return (lse - own) * has, lse, alpha * torch.mm(g, V.t().contiguous()), alpha * torch.mm(X.t().contiguous(), g), g.sum(0)


def _far(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("M,N,K,layout", [(66000, 300, 24, "feature"), (9000, 20000, 24, "feature"), (9000, 17001, 33, "unit")])
def test_pieces_of_the_classes_and_rows(M, N, K, layout):
    # more documents than one launch's pairs; more classes than a piece of g holds (2^27 bytes)
    x, W, labels, bias, dloss = _inputs(M, N, K, "bf16", layout)
    loss, lse = som.som_cross_entropy(x, W, labels, bias)
    dx, dW, dbias = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    want = _double(x, W, labels, bias, 1.0, dloss)
    # norms of many rounded values: each within its half step (2^-8) and a rounded g's (2^-8) at
    # the most, so the whole within 2^-7; the fp32 outputs within 2^-17
    for got, w, tol in zip((loss, lse, dx, dW, dbias), want, (2.0 ** -17, 2.0 ** -17, 2.0 ** -7, 2.0 ** -7, 2.0 ** -17)):
        assert _far(got, w) <= tol
    assert float((lse.double() - want[1]).abs().max()) < 1e-4
    # the rows one by one near the seams
    for i in (0, min(65535, M - 2), min(65536, M - 2), M - 1):
        one = som.som_cross_entropy(x[i:i + 1], W, labels[i:i + 1], bias)
        assert abs(float(one[1]) - float(lse[i])) < 1e-5
    assert bool((dx.float()[labels < 0] == 0).all())


# (unsplit; the scores' and dx's k axis split; more than one piece of the classes)
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("M,N,K", sorted(CLASSES))
def test_what_rounding_takes_from_a_codebooks_gradient_comes_back(M, N, K, pad, layout, kind):
    """dx of classes that have a mean mu in common.  Its own rounding leaves e of it.  g's roundings are of the
    same size relative to g, and leave e |g| |W - mu| and their sum times mu, where dx itself is |g| |W -
    mu| in size (the rows of g sum to zero): with uniform weights |mu|^2 = 3 |W - mu|^2, so e sqrt(1 + 1 +
    3) = 2.2 e in all, e sqrt(2) = 1.4 e where the sum comes back, and e sqrt(1 + 1 + 4 * 3) = 3.7 e where
    it is added with the wrong sign.  The limit lies between the first two, 1.7 e (of 24 features and
    few documents the sizes are off by up to a tenth)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(M)
    Wu = torch.rand((N, K), generator=g, device=DEV)
    Wm = Wu if layout == "unit" else Wu.t()
    W = torch.full((Wm.shape[0], Wm.shape[1] + pad), float("nan"), device=DEV).to(T[kind])[:, :Wm.shape[1]]
    W.copy_(Wm)
    W = W.t() if layout == "unit" else W
    t = 16.0 / K
    W64 = W.double().contiguous()
    labels = torch.randint(0, N, (M,), generator=g, device=DEV)
    x = (W64.t()[labels].float() + 0.3 * torch.randn((M, K), generator=g, device=DEV)).to(T[kind])
    labels[torch.rand(M, generator=g, device=DEV) < 0.1] = -1
    labels = labels.int()
    bias = (-t * (W64 * W64).sum(0)).float()
    dloss = 0.5 + torch.rand(M, generator=g, device=DEV)
    lse = som.som_cross_entropy(x, W, labels, bias, 2.0 * t)[1]
    dx = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias, 2.0 * t, need_dW=False, need_dbias=False)[0]
    _, _, want, _, _ = _double(x, W, labels, bias, 2.0 * t, dloss)
    own = _far(want.to(T[kind]), want)
    assert _far(dx, want) <= 1.7 * own
    # and it would be more without: g rounded as documented, its sums not put back
    has = (labels >= 0).double()
    v = torch.exp(2.0 * t * torch.mm(x.double(), W64) + bias.double() - lse.double()[:, None])
    v[torch.arange(M, device=DEV), labels.clamp(min=0).long()] -= 1.0
    v *= (dloss.double() * has)[:, None]
    size = 2.0 ** (14 if kind == "f16" else 0)              # dloss's largest is in [1, 2)
    rounded = (v * size).to(T[kind]).double() / size
    assert _far((2.0 * t * torch.mm(rounded, W64.t().contiguous())).to(T[kind]), want) > 1.9 * own


def _left_out(M, N, K, kind, layout, out, junk, mask, seed=0):
    """dx, dW and dbias where the classes `out` have a bias of `mask` and weights of `junk`, and the same in 64
    bits of the other classes alone (placed among zeros)."""
    x, W, labels, bias, dloss = _inputs(M, N, K, kind, layout, seed=seed, ignored=0.1)
    inside = torch.nonzero(~out)[:, 0].int()
    labels = torch.where((labels >= 0) & (labels < N), inside[labels.clamp(0, N - 1).long() % len(inside)], labels)
    bias[out] = mask
    W[:, out] = junk
    lse = som.som_cross_entropy(x, W, labels, bias)[1]
    got = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    number = torch.full((N,), -1, dtype=torch.int32, device=DEV)
    number[inside.long()] = torch.arange(len(inside), dtype=torch.int32, device=DEV)
    has = (labels >= 0) & (labels < N)
    mine = torch.where(has, number[labels.clamp(0, N - 1).long()], -1)
    want = _double(x, W[:, ~out], mine, bias[~out], 1.0, dloss)
    dW, dbias = torch.zeros((K, N), dtype=torch.float64, device=DEV), torch.zeros(N, dtype=torch.float64, device=DEV)
    dW[:, ~out], dbias[~out] = want[3], want[4]
    return got, (want[2], dW, dbias)


# (seeds whose weights' mean over the few classes is large by chance in some feature)
@pytest.mark.parametrize("M,N,K,kind,layout,pad,spread,alpha,with_bias,seed", [
    (117, 3, 411, "bf16", "feature", 8, 3.0, 1.0, True, 1534),
    (510, 9, 320, "bf16", "unit", 3, 1.0, 2.0, True, 2012),
    (257, 5, 4, "f16", "unit", 3, 3.0, 2.0, True, 9194),
    (24, 6, 384, "bf16", "unit", 0, 3.0, 1.0, True, 8729),
    (128, 12, 129, "f16", "unit", 1, 3.0, 2.0, True, 8479),
])
def test_few_classes_have_nothing_in_common_by_chance(M, N, K, kind, layout, pad, spread, alpha, with_bias, seed):
    x, W, labels, bias, dloss = _inputs(M, N, K, kind, layout, pad=pad, seed=seed, spread=spread)
    _check(x, W, labels, bias if with_bias else None, dloss, alpha, kind)


# (one launch of the scores, and a split k axis)
@pytest.mark.parametrize("M,N,K", [(300, 1000, 128), (60, 700, 4096)])
@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("mask", [float("-inf"), -1e30])
def test_weights_of_classes_that_are_left_out_do_not_reach_dx(mask, kind, layout, M, N, K):
    # the output's rounding and g's, each of its own size (see above): e sqrt(2), and less than 1.7 e
    out = torch.arange(N, device=DEV) % 3 == 0
    (dx, dW, dbias), want = _left_out(M, N, K, kind, layout, out, 2.0 ** 15, mask)
    for got, w in ((dx, want[0]), (dW, want[1])):
        assert _far(got, w) <= 1.7 * _far(w.to(T[kind]), w) + 2.0 ** -16
    assert _far(dbias, want[2]) <= 2.0 ** -16


# (one launch of the scores, and a split k axis; the last classes share their tile with none)
@pytest.mark.parametrize("M,N,K", [(300, 1000, 128), (60, 701, 4096)])
@pytest.mark.parametrize("layout", ["feature", "unit"])
def test_scores_of_classes_that_are_left_out_may_overflow(layout, M, N, K):
    x, W, labels, bias, dloss = _inputs(M, N, K, "bf16", layout, ignored=0.1)
    out = (torch.arange(N, device=DEV) % 3 == 0) | (torch.arange(N, device=DEV) >= N - 5)
    inside = torch.nonzero(~out)[:, 0].int()
    labels = torch.where((labels >= 0) & (labels < N), inside[labels.clamp(0, N - 1).long() % len(inside)], labels)
    labels[0] = 3                                    # a label that is left out
    bias[out] = float("-inf")
    W[:, out] = 0.0
    want = som.som_cross_entropy(x, W, labels, bias)
    want += som.som_cross_entropy_backward(dloss, x, W, labels, want[1], bias)
    assert all(bool(t.isfinite().all()) for t in want[1:])
    labels[0], W[:, out] = int(inside[0]), 3e38
    want = som.som_cross_entropy(x, W, labels, bias)
    assert all(bool(t.isfinite().all()) for t in want)
    got = som.som_cross_entropy_backward(dloss, x, W, labels, want[1], bias)
    W[:, out] = 0.0
    want = som.som_cross_entropy_backward(dloss, x, W, labels, want[1], bias)
    for a, b in zip(got, want):
        assert bool(a.isfinite().all()) and torch.equal(a, b)


@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_a_class_of_large_weights_moves_its_own_documents_alone(kind, layout):
    M, N, K = 400, 200, 96
    x, W, labels, bias, dloss = _inputs(M, N, K, kind, layout, ignored=0.1)
    labels = torch.where(labels == 77, 78, labels)
    labels[9] = 77
    W[:, 77] = 3e4
    bias[77] = -1e9                                  # no other document's
    dloss = dloss * M                                # (dx among fp16's normal numbers)
    lse = som.som_cross_entropy(x, W, labels, bias)[1]
    dx = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)[0]
    want = _double(x, W, labels, bias, 1.0, dloss)[2]
    rest = torch.arange(M, device=DEV) != 9
    assert _far(dx[rest], want[rest]) <= 1.7 * _far(want[rest].to(T[kind]), want[rest])
    assert _far(dx[9:10], want[9:10]) <= 2 * HALF[kind]


# (documents up to the most whose labels' roundings are kept, and one more; classes that several documents are
# labelled with; split axes, and more than one piece of the classes)
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("M,N,K", [(1, 900, 700), (2, 5000, 520), (5, 3001, 333), (17, 700, 2000), (64, 640, 1280),
                                   (100, 40000, 64), (150, 500000, 24), (255, 2000, 6000), (256, 1120, 512), (257, 3000, 128)])
def test_gradients_of_few_documents_are_as_near_as_their_rounding(M, N, K, pad, layout, kind):
    """A document's g is mostly its label's entry, one rounding of which reaches all of its row of dx and of
    its class in dW: of few documents these do not average out (two times the outputs' own rounding for one). Kept
    and multiplied, they leave the other entries', whose sum of squares is below a hundredth of the label's here (more
    than 600 classes, scores within 4 of each other): sqrt(1 + 0.01) of the own rounding, which of K and more
    elements is known within a tenth.  More documents go without: sqrt(2), within 1.55."""
    x, W, labels, bias, dloss = _inputs(M, N, K, kind, layout, pad=pad, seed=5, ignored=0.0 if M < 5 else 0.1)
    labels[M // 2:] = torch.where(labels[M // 2:] >= 0, labels[M // 2:] % max(1, N // 3), -1)
    if M > 20:
        labels[10:20] = 7                             # a class of many documents
    if M < 5:
        labels = labels.clamp(0, N - 1)
    dloss = dloss * M
    lse = som.som_cross_entropy(x, W, labels, bias)[1]
    got = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    want = _double(x, W, labels, bias, 1.0, dloss)[2:]
    limit = 1.11 if M <= 256 else 1.55
    for a, w in zip(got[:2], want[:2]):
        assert _far(a, w) <= limit * _far(w.to(T[kind]), w), (_far(a, w), _far(w.to(T[kind]), w))
    assert _far(got[2], want[2]) <= 2.0 ** -16
    again = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_gradients_against_differences():
    M, N, K = 6, 40, 16
    x, W, labels, bias, dloss = _inputs(M, N, K, "f16", "feature", ignored=0.0)
    labels = labels.clamp(max=N - 1)
    dloss = dloss * M
    _, lse = som.som_cross_entropy(x, W, labels, bias)
    dx, dW, dbias = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    xn, Wn, bn, ln, dn = _np(x), _np(W), _np(bias), labels.cpu().numpy(), _np(dloss)
    f = lambda a, b, c: float((oracle.cross_entropy(a, b, ln, c)[0] * dn).sum())  # noqa: E731
    h = 1e-5
    rng = np.random.default_rng(3)
    for got, which in ((dx, 0), (dW, 1), (dbias, 2)):
        base = (xn, Wn, bn)
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in base[which].shape)
            up, down = [a.copy() for a in base], [a.copy() for a in base]
            up[which][at] += h
            down[which][at] -= h
            want = (f(*up) - f(*down)) / (2 * h)
            # g and the result in fp16, sums of up to 40 terms of about one
            assert abs(float(got[at]) - want) <= 2.0 ** -9 * (abs(want) + 1.0)


def test_classes_left_out_and_rows_without_any():
    M, N, K = 70, 500, 64
    for layout in ("feature", "unit"):
        x, W, labels, bias, dloss = _inputs(M, N, K, "bf16", layout, ignored=0.0)
        labels = labels.clamp(max=N - 1)
        out = torch.zeros(N, dtype=torch.bool, device=DEV)
        out[::3] = True
        out[256:400] = True                      # a whole tile's columns of some shapes
        bias[out] = float("-inf")
        inside = torch.nonzero(~out)[:, 0].int()
        labels = inside[labels.long() % len(inside)]
        labels[5] = 0                            # a label that is left out
        loss, lse = som.som_cross_entropy(x, W, labels, bias)
        assert float(loss[5]) == float("inf") and bool(lse.isfinite().all())
        want, want_lse = oracle.cross_entropy(_np(x), _np(W), labels.cpu().numpy(), _np(bias))
        _near(lse, want_lse, 1e-4, "lse")
        _near(loss, want, 1e-4, "loss")
        dx, dW, dbias = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
        wx, wW, wb, _ = oracle.cross_entropy_backward(_np(dloss), _np(x), _np(W), labels.cpu().numpy(), _np(bias))
        keep = torch.ones(N, dtype=torch.bool, device=DEV)
        keep[0] = False
        assert bool((dbias[out & keep] == 0).all()) and bool((dW.float()[:, out & keep] == 0).all())
        assert _far(dx, torch.as_tensor(wx, device=DEV)) < 2.0 ** -7 and _far(dW, torch.as_tensor(wW, device=DEV)) < 2.0 ** -7
        assert _far(dbias, torch.as_tensor(wb, device=DEV)) < 2.0 ** -17
        # no class left at all
        bias[:] = float("-inf")
        loss, lse = som.som_cross_entropy(x, W, labels, bias)
        assert bool((lse == float("-inf")).all()) and bool((loss == float("inf")).all())
        for t in som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias):
            assert not t.any()
        for m in (1, 3, 20):                     # the kernels of few rows
            loss, lse = som.som_cross_entropy(x[:m], W, labels[:m], bias)
            assert bool((lse == float("-inf")).all()) and bool((loss == float("inf")).all())


@pytest.mark.parametrize("layout", ["feature", "unit"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_rows_that_count_for_nothing_may_hold_anything(bad, layout):
    M, N, K = 300, 700, 136
    x, W, labels, bias, dloss = _inputs(M, N, K, "f16", layout, ignored=0.3)
    has = (labels >= 0) & (labels < N)
    dloss[has.nonzero()[0, 0]] = 0.0
    none = ~has | (dloss == 0)
    _, lse = som.som_cross_entropy(x, W, labels, bias)
    want = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    dirty = x.clone()
    dirty[none, 3] = bad
    dirty[none.nonzero()[-1, 0]] = bad
    loss, lse = som.som_cross_entropy(dirty, W, labels, bias)
    assert bool((loss[~has] == 0).all()) and bool(lse[~none].isfinite().all())
    got = som.som_cross_entropy_backward(dloss, dirty, W, labels, lse, bias)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert not got[0][none].any()
    # a row that counts makes its own results NaN, and what all rows share
    i = int((~none).nonzero()[0, 0])
    dirty = x.clone()
    dirty[i, 0] = float("nan")
    loss, lse = som.som_cross_entropy(dirty, W, labels, bias)
    assert bool(loss[i].isnan()) and int(lse.isnan().sum()) == 1
    dx, dW, dbias = som.som_cross_entropy_backward(dloss, dirty, W, labels, lse, bias)
    assert bool(dx[i].isnan().all()) and torch.equal(dx[:i], want[0][:i]) and torch.equal(dx[i + 1:], want[0][i + 1:])
    assert bool(dbias.isnan().all())


def test_small_gradients_reach_fp16():
    # dloss of 2^-20 and probabilities of 1 / 4096: g is far below fp16's range, x is large
    M, N, K = 64, 4096, 64
    x, W, labels, bias, dloss = _inputs(M, N, K, "f16", "unit", ignored=0.0)
    labels = labels.clamp(max=N - 1)
    _, lse = som.som_cross_entropy(x, W, labels, None)
    one = som.som_cross_entropy_backward(torch.full((M,), 1.0, device=DEV), x, W, labels, lse)
    tiny = som.som_cross_entropy_backward(torch.full((M,), 2.0 ** -20, device=DEV), x, W, labels, lse)
    assert torch.equal(one[2] * 2.0 ** -20, tiny[2])
    # the same sums, rounded once to fp16's smallest step (2^-24) here and to 11 bits and then to
    # that step there: an 11-bit rounding is at most half a step of that size off a tie, so the two
    # are one step apart at the most
    for a, b in zip(one[:2], tiny[:2]):
        assert bool(b.any()) and bool(((a.double() * 2.0 ** -20).half().double() - b.double()).abs().max() <= 2.0 ** -24)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_loss_gradient_that_is_not_finite_leaves_the_other_documents_their_digits(bad):
    # (1 / 300 times a probability of 1 / 4096 is among fp16's last digits unless it is scaled)
    M, N, K = 300, 4096, 64
    x, W, labels, bias, dloss = _inputs(M, N, K, "f16", "unit", ignored=0.1)
    labels[7] = 11
    lse = som.som_cross_entropy(x, W, labels, bias)[1]
    _, _, want, _, _ = _double(x, W, labels, bias, 1.0, dloss)
    dloss[7] = bad
    dx, _, _ = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    rest = torch.arange(M, device=DEV) != 7
    # dx's rounding and g's (see above), and half of fp16's smallest step for each element of dx
    least = 2.0 ** -25 * (want[rest].numel() ** 0.5) / float(want[rest].norm())
    assert _far(dx[rest], want[rest]) <= 1.7 * _far(want[rest].half(), want[rest]) + least
    assert not bool(dx[7].isfinite().any())


def test_only_what_is_needed_and_given_outputs():
    M, N, K = 90, 333, 200
    x, W, labels, bias, dloss = _inputs(M, N, K, "bf16", "unit", pad=8)
    loss, lse = (torch.empty(M, device=DEV) for _ in range(2))
    got = som.som_cross_entropy(x, W, labels, bias, loss=loss, lse=lse)
    assert got[0] is loss and got[1] is lse
    full = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        part = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias, need_dx=need[0], need_dW=need[1],
                                              need_dbias=need[2])
        for a, b, n in zip(part, full, need):
            assert (a is None) if not n else torch.equal(a, b)
    wide = torch.full((M, K + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    wideW = torch.full((N, K + 24), 7.0, dtype=torch.bfloat16, device=DEV)
    dx, dW, _ = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias, dx=wide[:, :K], dW=wideW[:, :K].t())
    assert torch.equal(dx, full[0]) and torch.equal(dW, full[1])
    assert bool((wide[:, K:] == 7).all()) and bool((wideW[:, K:] == 7).all())


def test_empty_batches():
    x, W, labels, bias, dloss = _inputs(8, 50, 32, "f16", "feature")
    loss, lse = som.som_cross_entropy(x[:0], W, labels[:0], bias)
    assert loss.shape == lse.shape == (0,)
    dx, dW, dbias = som.som_cross_entropy_backward(dloss[:0], x[:0], W, labels[:0], lse, bias)
    assert dx.shape == (0, 32) and not dW.any() and not dbias.any()


def test_same_bits_again_and_on_streams_and_in_graphs():
    M, N, K = 300, 2500, 264
    x, W, labels, bias, dloss = _inputs(M, N, K, "bf16", "feature")
    loss, lse = som.som_cross_entropy(x, W, labels, bias)
    back = som.som_cross_entropy_backward(dloss, x, W, labels, lse, bias)
    again = som.som_cross_entropy(x, W, labels, bias)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = som.som_cross_entropy(x, W, labels, bias, stream=side)
    c = som.som_cross_entropy_backward(dloss, x, W, labels, b, bias, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, loss) and all(torch.equal(p, q) for p, q in zip(c, back))
    # captured with buffers of its own, replayed on new inputs, eager work between
    X, D, Lb = x.clone(), dloss.clone(), labels.clone()
    ws = torch.empty(som.som_cross_entropy_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(som.som_cross_entropy_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    out = [torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.empty_like(X), torch.empty((K, N), dtype=X.dtype, device=DEV),
           torch.empty(N, device=DEV)]

    def step():
        som.som_cross_entropy(X, W, Lb, bias, loss=out[0], lse=out[1], ws=ws)
        som.som_cross_entropy_backward(D, X, W, Lb, out[1], bias, dx=out[2], dW=out[3], dbias=out[4], ws=ws2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        X.copy_(x * (1.0 + 0.25 * k))
        D.copy_(dloss * (k + 1))
        Lb.copy_(labels.roll(k))
        graph.replay()
        torch.cuda.synchronize()
        wl, we = som.som_cross_entropy(X, W, Lb, bias)
        want = (wl, we, *som.som_cross_entropy_backward(D, X, W, Lb, we, bias))
        for p, q in zip(out, want):
            assert torch.equal(p, q), k


def test_refusals():
    x, W, labels, bias, dloss = _inputs(8, 50, 32, "f16", "feature")
    loss, lse = som.som_cross_entropy(x, W, labels, bias)
    fails = [(TypeError, lambda: som.som_cross_entropy(x.float(), W, labels)),
             (TypeError, lambda: som.som_cross_entropy(x, W.bfloat16(), labels)),
             (TypeError, lambda: som.som_cross_entropy(x, W, labels.long())),
             (ValueError, lambda: som.som_cross_entropy(x, W, labels[:7])),
             (ValueError, lambda: som.som_cross_entropy(x[:, :31], W, labels)),
             (ValueError, lambda: som.som_cross_entropy(x, W, labels, bias[:49])),
             (ValueError, lambda: som.som_cross_entropy(x, W, labels, lse=lse[:7])),
             (som.SomError, lambda: som.som_cross_entropy(x, W, labels, alpha=float("nan"))),
             (som.SomError, lambda: som.som_cross_entropy(x, W, None)),
             (som.SomError, lambda: som.som_cross_entropy(x, W, labels, ws=torch.empty(8, dtype=torch.uint8, device=DEV))),
             (ValueError, lambda: som.som_cross_entropy_backward(dloss[:7], x, W, labels, lse)),
             (ValueError, lambda: som.som_cross_entropy_backward(dloss, x, W, labels, lse[:7])),
             (TypeError, lambda: som.som_cross_entropy_backward(dloss.double(), x, W, labels, lse)),
             (TypeError, lambda: som.som_cross_entropy_backward(dloss, x, W, labels, lse, dx=x.float())),
             (ValueError, lambda: som.som_cross_entropy_backward(dloss, x, W, labels, lse, dx=x, need_dx=False)),
             (som.SomError, lambda: som.som_cross_entropy_backward(None, x, W, labels, lse))]
    for error, call in fails:
        with pytest.raises(error):
            call()
