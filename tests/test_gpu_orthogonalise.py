"""Orthogonalised updates on the GPU against the fp64 oracle.

Tolerance.  Every element of X, A and B that a product reads is rounded to 11 bits, uniformly:
r = 2^-11 / sqrt(3) of itself at the most (a rounding's root mean square is at most half a
step over sqrt 3).  Of a step's terms a X is exact, (b A + c A A) X carries the roundings of A, twice in
A A, of B and of X: their norms are at most |b| s^3 and c s^5 for singular values s up to 1.2, which
for (3.4445, -4.775, 2.0315) are 8.3 and 5.1, but cancel in X, so for directions of s = 1 the
terms are 4.8 and 2.0, their roundings r sqrt((4.8 + 2 * 2.0)^2 + 2.8^2 * 2) = 9.7 r, damped by the next
step's slope (a + 3 b s^2 + 5 c s^4 = -0.7 at s = 1, at most 1.5 between 0.7 and 1.2 in size): a
geometric sum of at most 2 of them in root mean square, 20 r = 5.6e-3 of the result in the worst
case that all directions are there; the result's own rounding is 2^-8 of each element.  Every test asks for
that; the typical error is a fifth (2e-3)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from dense_plan import MIRRORED, symmetric_tile  # noqa: E402
from oracle import train as oracle  # noqa: E402

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
QUINTIC, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)
WITHIN = 5.6e-3 + 2.0 ** -8 / 3 ** 0.5


def _view(values, dtype, pad):
    rows, cols = values.shape
    wide = torch.full((rows, cols + pad), float("nan"), device=DEV).to(dtype)
    wide[:, :cols] = torch.as_tensor(values, device=DEV).to(dtype)
    return wide[:, :cols]


def _far(got, want):
    return np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (5, 64), (64, 64), (65, 63), (63, 200), (100, 100), (128, 512), (300, 129),
          (257, 1000), (1030, 255), (520, 520)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalise(rows, cols, kind):
    rng = np.random.default_rng(rows * 100 + cols)
    pad = (rows + cols) % 3 * 3
    G = _view(rng.normal(size=(rows, cols)) * 1e-2, T[kind], pad)
    wide = torch.full((rows, cols + 5), 7.0, dtype=torch.bfloat16, device=DEV)
    for coefficients, steps in ((QUINTIC, 5), (QUINTIC, 1), (CUBIC, 3)):
        y = som.som_orthogonalise(G, steps, coefficients, y=wide[:, :cols])
        assert _far(y, oracle.orthogonalise(G.double().cpu().numpy(), steps, coefficients)) <= WITHIN
        assert bool((wide[:, cols:] == 7).all())


@pytest.mark.parametrize("rows,cols", [(256, 384), (384, 256)])
@pytest.mark.parametrize("spectrum", ["equal", "wide", "spikes", "one"])
def test_spectra(spectrum, rows, cols):
    rng = np.random.default_rng(rows)
    u, s, v = np.linalg.svd(rng.normal(size=(rows, cols)), full_matrices=False)
    k = len(s)
    s = {"equal": np.ones(k), "wide": np.logspace(0, -4, k), "spikes": np.r_[np.full(4, 30.0), np.ones(k - 4)],
         "one": np.r_[1.0, np.zeros(k - 1)]}[spectrum]
    G = torch.as_tensor(u @ np.diag(s) @ v, dtype=torch.float32, device=DEV)
    y = som.som_orthogonalise(G)
    assert _far(y, oracle.orthogonalise(G.double().cpu().numpy(), 5, QUINTIC)) <= WITHIN
    got = np.linalg.svd(y.double().cpu().numpy(), compute_uv=False)
    if spectrum in ("equal", "spikes"):
        assert 0.6 < got.min() and got.max() < 1.25


def test_many_cubic_steps_reach_an_orthogonal_matrix():
    rng = np.random.default_rng(0)
    G = torch.as_tensor(rng.normal(size=(64, 500)), dtype=torch.float32, device=DEV)
    y = som.som_orthogonalise(G, 20, CUBIC).double()
    gram = y @ y.t().contiguous()
    # y's elements are 2^-8 off at the most, its rows 2^-8 of their length of one; the steps' 2^-11 settle at s = 1
    assert float((gram - torch.eye(64, device=DEV, dtype=torch.float64)).abs().max()) < 3 * 2.0 ** -8


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1.0, 1e30, 1e38])
def test_sizes_whose_squares_leave_fp32(scale):
    rng = np.random.default_rng(1)
    G = torch.as_tensor(rng.uniform(-1, 1, size=(70, 90)), dtype=torch.float32, device=DEV)
    y = som.som_orthogonalise(G * scale)
    assert _far(y, oracle.orthogonalise((G * scale).double().cpu().numpy(), 5, QUINTIC)) <= WITHIN


def test_zeros_and_values_that_are_not_finite():
    for shape in ((1, 1), (70, 200), (300, 40)):
        G = torch.zeros(shape, device=DEV)
        assert not som.som_orthogonalise(G).any()
        for bad in (float("nan"), float("inf"), float("-inf")):
            G = torch.ones(shape, device=DEV)
            G[-1, -1] = bad
            assert bool(som.som_orthogonalise(G).isnan().all())


def test_large_and_in_place():
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    for rows, cols in ((1200, 2500), (2100, 2100)):
        G = torch.randn((rows, cols), generator=g, device=DEV).bfloat16()
        X = G.double() / torch.linalg.vector_norm(G.double())
        for _ in range(5):
            A = torch.mm(X, X.t().contiguous())
            X = QUINTIC[0] * X + torch.mm(QUINTIC[1] * A + QUINTIC[2] * torch.mm(A, A), X)
        y = som.som_orthogonalise(G)
        assert float((y.double() - X).norm() / X.norm()) < WITHIN
        back = som.som_orthogonalise(G.t().contiguous())
        assert float((back.double().t() - X).norm() / X.norm()) < WITHIN
        again = G.clone()
        assert som.som_orthogonalise(again, y=again) is again and torch.equal(again, y)


def test_streams_and_graphs():
    rng = np.random.default_rng(2)
    G = torch.as_tensor(rng.normal(size=(200, 333)), dtype=torch.float32, device=DEV)
    want = som.som_orthogonalise(G)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = som.som_orthogonalise(G, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want) and torch.equal(som.som_orthogonalise(G), want)
    X, y = G.clone(), torch.empty_like(want)
    ws = torch.empty(som.som_orthogonalise_workspace_bytes(200, 333), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        som.som_orthogonalise(X, y=y, ws=ws)
    for k in range(3):
        X.copy_(G.roll(k, 0) + 0.1 * k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, som.som_orthogonalise(X))


STEEP = (4.0848, -6.8946, 2.9270)          # |slope| up to 3.2 about s = 1: roundings grow with every step


def _own(want):
    """The result's own rounding."""
    return _far(torch.as_tensor(want).to(torch.bfloat16), want)


def _roundings(G, steps, coefficients, low, seed=0):
    """What the documented roundings leave of the result: X, A and B off by up to 2^-11 of each element (2^-25
    where that is more: fp16's subnormal step), uniformly, in 64 bits.  A rounding to 11 bits is off
    by 2^-11 at the most and by half of it where its leading digits are largest, so this is more
    than it leaves (1.4 times, for elements of all sizes alike)."""
    rng = np.random.default_rng(seed)
    a, b, c = coefficients
    G = G.T if G.shape[0] > G.shape[1] else G

    def off(v, symmetric):
        e = rng.uniform(-1.0, 1.0, v.shape) * np.maximum(2.0 ** -11 * np.abs(v), 2.0 ** -25 if symmetric else 0.0)
        return v + (np.triu(e) + np.triu(e, 1).T if symmetric else e)

    X = Y = G / np.linalg.norm(G)
    for _ in range(steps):
        h = off(X, False)
        A = off(h @ h.T, True)
        B = b * A + c * (A @ A)
        X = a * X + (B if low else off(B, True)) @ h
        S = Y @ Y.T
        Y = a * Y + (b * S + c * (S @ S)) @ Y
    return np.linalg.norm(X - Y) / np.linalg.norm(Y)


# (short sides above and up to 256, of the small products and of the large ones)
@pytest.mark.parametrize("rows,cols", [(300, 300), (153, 221), (600, 500), (1100, 600)])
@pytest.mark.parametrize("coefficients,steps", [(QUINTIC, 1), (QUINTIC, 5), (QUINTIC, 10), (QUINTIC, 30), (QUINTIC, 64),
                                                (STEEP, 3), (STEEP, 5), (STEEP, 8)])
def test_errors_grow_with_steps_and_slopes_as_roundings_do(coefficients, steps, rows, cols):
    # within a quarter more than the simulated roundings, which are of other draws, and y's own
    G = torch.as_tensor(np.random.default_rng(steps).normal(size=(rows, cols)), dtype=torch.float32, device=DEV)
    G64 = G.double().cpu().numpy()
    want = oracle.orthogonalise(G64, steps, coefficients)
    error = _roundings(G64, steps, coefficients, min(rows, cols) <= 256)
    assert _far(som.som_orthogonalise(G, steps, coefficients), want) <= np.hypot(1.25 * error, 1.01 * _own(want))


def _in_16_bits(G, steps, coefficients, low):
    """The steps with X, A and B rounded to fp16, and what that leaves of A and B multiplied too (low) or not."""
    a, b, c = coefficients
    tall = G.shape[0] > G.shape[1]
    X = (G.T if tall else G) / np.linalg.norm(G)
    size = 2.0 ** round(0.5 * np.log2(G.size))

    def half(v):
        return v.astype(np.float16).astype(np.float64)

    for _ in range(steps):
        h = half(X * size) / size
        A = half(h @ h.T)
        B = b * A + c * (A @ A)
        X = a * X + (B if low else half(B)) @ h
    return X.T if tall else X


@pytest.mark.parametrize("rows,cols", [(32, 1000), (100, 900), (900, 100)])
def test_what_rounding_leaves_of_the_polynomial_is_multiplied_too(rows, cols):
    G = torch.as_tensor(np.random.default_rng(rows).normal(size=(rows, cols)), dtype=torch.float32, device=DEV)
    G64 = G.double().cpu().numpy()
    want = oracle.orthogonalise(G64, 5, QUINTIC)
    size = np.linalg.norm(want)
    kept, dropped = (np.linalg.norm(_in_16_bits(G64, 5, QUINTIC, low) - want) / size for low in (True, False))
    # the same roundings but for those of fp32, which move a few of them; y's own is known to a hundredth
    limit = 1.02 * np.hypot(1.15 * kept, _own(want))
    assert np.hypot(dropped, _own(want)) > limit
    assert _far(som.som_orthogonalise(G), want) <= limit


# (both layouts; the last row and column of tiles are partial)
@pytest.mark.parametrize("rows,cols", sorted(MIRRORED))
def test_symmetric_products_in_the_largest_tiles(rows, cols):
    assert symmetric_tile(som.load(), rows, cols) == ("256x256", True)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    G = torch.randn((rows, cols), generator=g, device=DEV)
    X = G.double() / torch.linalg.vector_norm(G.double())
    X = X.t().contiguous() if rows > cols else X
    for _ in range(3):
        A = torch.mm(X, X.t().contiguous())
        X = QUINTIC[0] * X + torch.mm(QUINTIC[1] * A + QUINTIC[2] * torch.mm(A, A), X)
    X = X.t() if rows > cols else X
    y = som.som_orthogonalise(G, 3)
    assert float((y.double() - X).norm() / X.norm()) <= WITHIN
    # everywhere alike: no block of 32 x 32 has more than its share (a wrong one is off by its whole size,
    # an element by 2^-8 of itself and the typical error five times over)
    bad = (y.double() - X).abs() > 2.0 ** -8 * X.abs() + 5 * WITHIN * float(X.norm()) / (rows * cols) ** 0.5
    assert int(bad.sum()) <= 1e-4 * rows * cols and not bool(_blocks_mean(bad.float()).gt(0.1).any())


def _blocks_mean(v):
    return torch.nn.functional.avg_pool2d(v[None, None], 32, ceil_mode=True, count_include_pad=False)[0, 0]


def test_refusals():
    G = torch.zeros((8, 16), device=DEV)
    c = som.som_orthogonalise
    fails = [(som.SomError, lambda: c(G, 0)), (som.SomError, lambda: c(G, 65)), (som.SomError, lambda: c(G[:0])),
             (som.SomError, lambda: c(G, 5, (float("nan"), 0.0, 0.0))), (som.SomError, lambda: c(G, 5, (65.0, 0.0, 0.0))),
             (TypeError, lambda: c(G.double())), (TypeError, lambda: c(G, y=G)), (ValueError, lambda: c(G.t())),
             (ValueError, lambda: c(G, y=torch.empty((8, 15), dtype=torch.bfloat16, device=DEV))),
             (ValueError, lambda: c(G, 5, (1.0, 2.0))),
             (som.SomError, lambda: c(G, ws=torch.empty(64, dtype=torch.uint8, device=DEV)))]
    for error, call in fails:
        with pytest.raises(error):
            call()
