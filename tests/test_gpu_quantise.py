"""Blocks of 8 bits on the GPU against the fp64 oracle: a factor is rounded once (a division, 2^-24
of itself); a code stands for its value within half a step of E4M3 (2^-4 of it, or 2^-10 factors
below 2^-6 of them) and the 2^-22 of the factor's inverse and the product with it."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import train as oracle  # noqa: E402

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SHAPES = [(1, 1), (1, 127), (3, 128), (2, 129), (16, 512), (17, 513), (127, 130), (128, 128), (129, 300), (300, 1023), (5, 4100)]


def _x(rows, cols, kind, pad, seed=0):
    rng = np.random.default_rng(rows * 1009 + cols + seed)
    wide = torch.full((rows, cols + pad), float("nan"), device=DEV).to(T[kind])
    values = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=(1, cols)))
    wide[:, :cols] = torch.as_tensor(values, device=DEV).to(T[kind])
    return wide[:, :cols]


def _check(x, block_rows, transpose, q, scale):
    want = x.double().cpu().numpy()
    want = want.T if transpose else want
    factor = oracle.quantise_scale(want, block_rows)
    got = scale.double().cpu().numpy()
    assert got.shape == factor.shape and (np.abs(got - factor) <= 2.0 ** -24 * factor + 2.0 ** -150).all()
    each = oracle.spread(got, *want.shape, block_rows)
    value = q.double().cpu().numpy() * each
    assert (np.abs(value - want) <= np.abs(want) * (2.0 ** -4 + 2.0 ** -22) + 2.0 ** -10 * each).all()
    # the largest of a block takes the largest code
    top = np.abs(q.double().cpu().numpy())
    assert oracle.quantise_scale(top, block_rows).max() <= 1.0


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantise(rows, cols, transpose, block_rows, kind):
    x = _x(rows, cols, kind, (rows + cols) % 3 * 3)
    qr, qc = (cols, rows) if transpose else (rows, cols)
    wide = torch.full((qr, qc + 5), 1.0, device=DEV).to(torch.float8_e4m3fn)
    q, scale = som.som_quantise(x, block_rows, transpose, q=wide[:, :qc])
    _check(x, block_rows, transpose, q, scale)
    assert bool((wide[:, qc:].float() == 1.0).all())
    # factors laid out the other way, and codes of their own
    other = torch.full((scale.shape[0], scale.shape[1] + 3), 9.0, device=DEV)
    q2, s2 = som.som_quantise(x, block_rows, transpose, scale=other[:, :scale.shape[1]])
    assert torch.equal(q2.view(torch.uint8), q.contiguous().view(torch.uint8)) and torch.equal(s2, scale)
    assert bool((other[:, scale.shape[1]:] == 9.0).all())


def test_the_transpose_of_square_blocks_is_the_same_blocks():
    x = _x(300, 700, "bf16", 0)
    q, s = som.som_quantise(x, 128)
    qt, st = som.som_quantise(x, 128, True)
    assert torch.equal(qt.view(torch.uint8).t(), q.view(torch.uint8)) and torch.equal(st.t(), s)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("block_rows,transpose", [(1, False), (1, True), (128, False), (128, True)])
def test_blocks_of_nothing_and_next_to_it(kind, block_rows, transpose):
    x = torch.zeros((130, 400), device=DEV)
    x[0, 5], x[129, 399] = 1e-40, 3.0
    x[64, 200] = 2.0 ** -120
    x = x.to(T[kind])
    q, scale = som.som_quantise(x, block_rows, transpose)
    _check(x, block_rows, transpose, q, scale)
    assert bool((scale > 0).all()) and bool(q.float().isfinite().all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("block_rows,transpose", [(1, False), (1, True), (128, False), (128, True)])
def test_not_finite_values_spoil_their_block_alone(bad, block_rows, transpose):
    x = _x(260, 300, "f16", 0)
    clean_q, clean = som.som_quantise(x, block_rows, transpose)
    x[130, 140] = bad
    q, scale = som.som_quantise(x, block_rows, transpose)
    spoilt = ~scale.isfinite()
    assert int(spoilt.sum()) == 1
    assert torch.equal(scale[~spoilt], clean[~spoilt])
    each = torch.as_tensor(oracle.spread(scale.double().cpu().numpy(), *q.shape, block_rows), device=DEV)
    value = q.double() * each
    assert bool((value.isfinite() == each.isfinite()).all())
    same = q.view(torch.uint8) == clean_q.view(torch.uint8)
    assert bool(same[each.isfinite()].all())


def _division(x, scale, block_rows):
    """The codes of x / s: fp32's quotient, rounded to E4M3, by the host."""
    each = scale.cpu().repeat_interleave(128, 1)[:, :x.shape[1]].repeat_interleave(block_rows, 0)[:x.shape[0]]
    return (x.float().cpu() / each).to(torch.float8_e4m3fn)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("block_rows,transpose", [(1, False), (1, True), (128, False), (128, True)])
def test_codes_are_the_quotients(kind, block_rows, transpose):
    # every block of 128 x 128 of a size of its own, over the type's range, with zeros of both signs
    # (two such matrices, whose quotients are next to a tie between two codes for many values)
    small, large = {"f32": (-148, 118), "f16": (-20, 10), "bf16": (-132, 118)}[kind]
    for seed in (0, 1):
        x = _x(1100, 1000, kind, 0, seed).float()
        size = torch.as_tensor(np.random.default_rng(seed).integers(small, large, (9, 8)), device=DEV)
        half = (size // 2).repeat_interleave(128, 0).repeat_interleave(128, 1)[:1100, :1000]
        rest = (size - size // 2).repeat_interleave(128, 0).repeat_interleave(128, 1)[:1100, :1000]
        x = (torch.ldexp(torch.ldexp(x, half), rest)).to(T[kind])
        x[::7, ::5] = 0.0
        x[::11, ::3] = -0.0
        q, scale = som.som_quantise(x, block_rows, transpose)
        want = _division(x.t() if transpose else x, scale, block_rows)
        assert bool(scale.isfinite().all())
        differ = q.cpu().view(torch.uint8) != want.view(torch.uint8)
        assert not bool(differ.any()), (int(differ.sum()), differ.nonzero()[:4].tolist())


def test_many_rows_and_columns():
    x = torch.randn((70000, 136), device=DEV).bfloat16()
    # in 64 bits: torch divides an fp32 tensor by a number as a product with its rounded inverse
    want = torch.nn.functional.pad(x.double().abs(), (0, 120)).view(70000, 2, 128).amax(2) / 448.0
    for scale in (som.som_quantise(x)[1], som.som_quantise(x.t().contiguous(), 1, True)[1]):
        assert bool(((scale.double() - want).abs() <= 2.0 ** -24 * want).all())


def test_streams_and_graphs():
    x = _x(200, 600, "bf16", 0)
    want = som.som_quantise(x, 1, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = som.som_quantise(x, 1, True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got[1], want[1])
    X, q, s = x.clone(), torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        som.som_quantise(X, 1, True, q=q, scale=s)
    for k in range(3):
        X.copy_(x * (1.5 + k))
        graph.replay()
        torch.cuda.synchronize()
        want = som.som_quantise(X, 1, True)
        assert torch.equal(q.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s, want[1])


def test_refusals():
    x = _x(8, 256, "f16", 0)
    s = torch.empty((8, 2), device=DEV)
    assert som.som_quantise(x[:0])[0].shape == (0, 256)
    fails = [(ValueError, lambda: som.som_quantise(x, 2)), (TypeError, lambda: som.som_quantise(x.double())),
             (ValueError, lambda: som.som_quantise(x, q=torch.empty((8, 255), device=DEV).to(torch.float8_e4m3fn))),
             (TypeError, lambda: som.som_quantise(x, q=torch.empty((8, 256), dtype=torch.uint8, device=DEV))),
             (ValueError, lambda: som.som_quantise(x, scale=s[:, :1])), (TypeError, lambda: som.som_quantise(x, scale=s.double())),
             (som.SomError, lambda: som.som_quantise(x, scale=s[:1].expand(8, 2))),
             (som.SomError, lambda: som.som_quantise(x, scale=torch.empty(9, device=DEV).as_strided((8, 2), (1, 1)))),
             (ValueError, lambda: som.som_quantise(x.t()))]
    for error, call in fails:
        with pytest.raises(error):
            call()
