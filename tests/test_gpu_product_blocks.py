"""The product of operands in blocks of 8 bits on the GPU against the fp64 oracle.

Tolerances (u = 2^-24, t = half a unit of the output's type), of a sum of magnitudes S over
blocks of 128 products, each times its two factors:
  y of 16 bits: the matrix instruction lines a block's products up and cuts each by 2^-21 of the
  largest at the most, 128 of them 2^-14 of S (measured: 2^-15.8 of a block's, at the worst);
  y of 32 bits, and up to four rows: 2 * 128 u of S for the block's sum;
  factors and the sum of blocks: (K / 128 + 8) u of S; activation 2^-17 of what it gives, and its slope
  (at most 1.13) times the argument's error; the output t of itself."""

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
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}
U = 2.0 ** -24


def _np(t):
    return t.double().cpu().numpy()


def _near(got, want, tol, what=""):
    got = _np(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4],
                           np.broadcast_to(tol, want.shape)[bad][:4])


def _codes(rows, cols, pad, rng, spread=1.0):
    """Codes of E4M3 in a wider array whose other columns are NaN."""
    wide = torch.full((rows, cols + pad), float("nan"), device=DEV).to(torch.float8_e4m3fn)
    v = torch.as_tensor(rng.normal(size=(rows, cols)) * 100.0 * spread, device=DEV).clamp(-448, 448)
    wide[:, :cols] = v.to(torch.float8_e4m3fn)
    return wide[:, :cols]


def _factors(rows, K, block_rows, by_block, rng):
    shape = (-(-rows // block_rows), -(-K // 128))
    v = torch.as_tensor(np.exp(rng.normal(size=shape)) * 0.01, dtype=torch.float32, device=DEV)
    return v.t().contiguous().t() if by_block else v


def _want(x, xs, W, ws, x_rows, w_rows, alpha, out, few, bias=None, act="none", residual=None):
    M, K = x.shape
    N = W.shape[1]
    fx, fw = oracle.spread(_np(xs), M, K, x_rows), oracle.spread(_np(ws), N, K, w_rows)
    xn, Wn = _np(x), _np(W).T
    y, pre = oracle.product_blocks(xn, fx, Wn, fw, bias, act, residual, alpha)
    S = abs(alpha) * ((np.abs(xn) * fx) @ (np.abs(Wn) * fw).T)
    calc = S * ((256 * U if out == "f32" or few else 2.0 ** -14) + (K / 128 + 8) * U)
    if bias is not None:
        calc = calc + 2 * U * (np.abs(bias) + S)
    return y, pre, calc


SHAPES = [(1, 1, 1), (1, 17, 128), (2, 16, 129), (3, 130, 1000), (4, 257, 272), (5, 129, 127), (7, 300, 4100), (16, 128, 128),
          (17, 1, 300), (33, 127, 256), (64, 512, 1024), (65, 200, 15), (100, 333, 641), (129, 129, 2000), (200, 2047, 520),
          (257, 255, 384), (300, 1000, 96), (1030, 1100, 260), (20, 130, 9000)]


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K, w_rows, out):
    rng = np.random.default_rng(M * 31 + N * 7 + K)
    for pad, by_block, x_rows in ((-K % 16, True, 1), ((M + N) % 5, False, 128 if M > 1 else 1)):
        x, W = _codes(M, K, pad, rng), _codes(N, K, pad, rng).t()
        xs, ws = _factors(M, K, x_rows, by_block, rng), _factors(N, K, w_rows, not by_block, rng)
        y, _, calc = _want(x, xs, W, ws, x_rows, w_rows, 1.0, out, M <= 4)
        wide = torch.full((M, N + 3), 7.0, device=DEV).to(T[out])
        got = som.som_product_blocks(x, xs, W, ws, y=wide[:, :N])
        _near(got, y, calc + np.abs(y) * HALF[out] + TINY[out])
        assert bool((wide[:, N:] == 7).all())


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M,N,K", [(1, 70, 300), (30, 300, 700), (300, 520, 1100), (17, 100, 9000)])
def test_epilogue(M, N, K, act, out):
    rng = np.random.default_rng(M + N)
    x, W = _codes(M, K, 0, rng, 0.05), _codes(N, K, 0, rng, 0.05).t()
    xs, ws = _factors(M, K, 1, True, rng), _factors(N, K, 128, True, rng)
    bias = torch.as_tensor(rng.normal(size=N), dtype=torch.float32, device=DEV)
    res = torch.as_tensor(rng.normal(size=(M, N)), device=DEV).to(T[out])
    y, pre, calc = _want(x, xs, W, ws, 1, 128, 3.0, out, M <= 4, _np(bias), act, _np(res))
    kept = torch.empty((M, N), dtype=T[out], device=DEV)
    got = som.som_product_blocks(x, xs, W, ws, bias=bias, act=act, residual=res, alpha=3.0, dtype=T[out], pre=kept)
    _near(kept, pre, calc + np.abs(pre) * HALF[out] + TINY[out], "pre")
    _near(got, y, 1.13 * calc + 2.0 ** -17 * np.abs(y - _np(res)) + 2.0 ** -20 * np.abs(pre) + np.abs(y) * HALF[out]
          + 2 * U * np.abs(_np(res)) + TINY[out], "y")


def test_large_tiles():
    # every shape of tile, rows and columns that end inside them, steps from one to many
    rng = np.random.default_rng(5)
    for M, N, K in ((4100, 3900, 256), (2050, 2300, 1290), (1500, 700, 384), (520, 4000, 128), (700, 600, 4000)):
        x, W = _codes(M, K, -K % 16, rng), _codes(N, K, -K % 16, rng).t()
        for w_rows in (128, 1):
            xs, ws = _factors(M, K, 1, True, rng), _factors(N, K, w_rows, True, rng)
            for out in ("f16", "f32"):
                # (the oracle in 64 bits on the device)
                col = torch.arange(K, device=DEV) // 128
                a, b = x.double() * xs.double()[:, col], W.t().double() * ws.double()[torch.arange(N, device=DEV) // w_rows][:, col]
                want, S = torch.mm(a, b.t().contiguous()), torch.mm(a.abs(), b.abs().t().contiguous())
                got = som.som_product_blocks(x, xs, W, ws, dtype=T[out], alpha=2.0 ** -6)
                want, S = want / 64, S / 64
                tol = S * ((256 * U if out == "f32" else 2.0 ** -14) + (K / 128 + 8) * U) + want.abs() * HALF[out] + TINY[out]
                bad = (got.double() - want).abs() > tol
                assert not bool(bad.any()), (M, N, K, w_rows, out, int(bad.sum()), bad.nonzero()[:4].tolist())


def test_codes_of_every_kind():
    # every code beside others: subnormal and largest values, zeros of both signs; NaN stays in its row and column
    codes = torch.arange(256, dtype=torch.uint8, device=DEV)
    codes = codes[(codes & 127) != 127]
    x = codes.repeat(40)[: 38 * 254].view(38, 254)[:, :250].contiguous().view(torch.float8_e4m3fn)
    W = codes.flip(0).repeat(140)[: 135 * 254].view(135, 254)[:, :250].contiguous().view(torch.float8_e4m3fn).t()
    rng = np.random.default_rng(1)
    for w_rows in (1, 128):
        xs, ws = _factors(38, 250, 1, True, rng), _factors(135, 250, w_rows, True, rng)
        for out in ("bf16", "f32"):
            y, _, calc = _want(x, xs, W, ws, 1, w_rows, 1.0, out, False)
            _near(som.som_product_blocks(x, xs, W, ws, dtype=T[out]), y, calc + np.abs(y) * HALF[out])
    bad = x.view(torch.uint8).clone()
    bad[5, 200] = 127
    y = som.som_product_blocks(bad.view(torch.float8_e4m3fn), xs, W, ws)
    assert bool(y[5].isnan().all()) and int(y.isnan().sum()) == 135
    clean = som.som_product_blocks(x, xs, W, ws)
    assert torch.equal(y[:5], clean[:5]) and torch.equal(y[6:], clean[6:])
    # a factor that is not finite spoils its rows (or units) alone
    for w_rows in (1, 128):
        ws = _factors(135, 250, w_rows, True, rng)
        clean = som.som_product_blocks(x, xs, W, ws)
        ws[0, 1] = float("nan")
        y = som.som_product_blocks(x, xs, W, ws)
        assert bool(y[:, :w_rows].isnan().all()) and torch.equal(y[:, w_rows:], clean[:, w_rows:])


def _cuts(x, sx, x_rows, W, sw, w_rows):
    """The most that cutting takes from each sum: of eight consecutive k seven products (the largest has no
    digits to lose: the codes' product has eight) by a unit each of 2^-13 of the power of two that the
    largest pair of exponents gives, times the block's factors."""
    M, K = x.shape
    N = W.shape[1]

    def powers(codes):
        e = torch.floor(torch.log2(codes.double().abs().clamp(min=2.0 ** -6)))         # subnormal codes: the least
        e = torch.where(codes.double() == 0, torch.full_like(e, -100.0), e)
        return torch.nn.functional.pad(e, (0, -K % 8), value=-100.0).view(len(e), -1, 8)

    a, b = powers(x), powers(W.t())
    cut = torch.zeros((M, N), dtype=torch.float64, device=DEV)
    for group in range(a.shape[1]):
        largest = (a[:, None, group] + b[None, :, group]).amax(2)
        block = group * 8 // 128
        factors = (sx.double()[torch.arange(M, device=DEV) // x_rows, block][:, None]
                   * sw.double()[torch.arange(N, device=DEV) // w_rows, block][None])
        cut += 7 * 2.0 ** -13 * torch.exp2(largest) * factors
    return cut


@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("kind", ["normal", "columns", "one column", "heavy", "few digits"])
@pytest.mark.parametrize("M,N,K", [(90, 140, 14), (130, 70, 128), (64, 129, 1000)])
def test_products_far_below_the_largest_of_eight_are_cut_as_documented(M, N, K, kind, w_rows, out):
    rng = np.random.default_rng(M + N + K)
    x, W = rng.normal(size=(M, K)), rng.normal(size=(N, K))
    if kind == "columns":
        x *= np.exp(2.0 * rng.normal(size=(1, K)))
    elif kind == "one column":
        x[:, ::16] *= 300.0
    elif kind == "heavy":
        x, W = rng.standard_t(1.5, size=(M, K)), rng.standard_t(1.5, size=(N, K))
    elif kind == "few digits":             # the sum is what is left of two large products
        x[:, 0::8], x[:, 1::8] = 1000.0, 1000.0
        W[:, 1::8] = -W[:, 0::8][:, :W[:, 1::8].shape[1]]
    qx, sx = som.som_quantise(torch.as_tensor(x, dtype=torch.float32, device=DEV))
    qW, sW = som.som_quantise(torch.as_tensor(W, dtype=torch.float32, device=DEV) * K ** -0.5, w_rows)
    y, _, calc = _want(qx, sx, qW.t(), sW, 1, w_rows, 1.0, "f32", False)
    cut = _np(_cuts(qx, sx, 1, qW.t(), sW, w_rows))
    got = som.som_product_blocks(qx, sx, qW.t(), sW, dtype=T[out], alpha=2.0 ** -8)
    want = y / 256
    _near(got, want, (cut + calc) / 256 * (1 + HALF[out]) + np.abs(want) * HALF[out] + TINY[out])
    # into fp32 nothing is cut
    got = som.som_product_blocks(qx, sx, qW.t(), sW, dtype=torch.float32, alpha=2.0 ** -8)
    _near(got, want, calc / 256 + np.abs(want) * HALF["f32"])


def test_quantised_products_and_their_gradients():
    """Forward, dx and dW of a projection, all in blocks of 8 bits, against the same of the codes' values."""
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    M, K, N = 330, 520, 270
    x, W, dy = (torch.randn(s, generator=g, device=DEV).bfloat16() for s in ((M, K), (N, K), (M, N)))
    qx, sx = som.som_quantise(x)
    qW, sW = som.som_quantise(W, 128)
    qWt, sWt = som.som_quantise(W, 128, transpose=True)
    qd, sd = som.som_quantise(dy)
    qdt, sdt = som.som_quantise(dy, transpose=True)
    qxt, sxt = som.som_quantise(x, transpose=True)

    def check(got, a, fa, b, fb, rows):
        y, _, calc = _want(a, fa, b.t(), fb, 1, rows, 1.0, "bf16", False)
        _near(got, y, calc + np.abs(y) * HALF["bf16"])

    check(som.som_product_blocks(qx, sx, qW.t(), sW), qx, sx, qW, sW, 128)
    check(som.som_product_blocks(qd, sd, qWt.t(), sWt), qd, sd, qWt, sWt, 128)             # dx = dy W
    check(som.som_product_blocks(qdt, sdt, qxt.t(), sxt), qdt, sdt, qxt, sxt, 1)           # dW = dy^T x, by unit
    # and near the unquantised ones: an operand's codes are 2^-4 off at the most, uniformly 2^-5.8
    for got, want in ((som.som_product_blocks(qx, sx, qW.t(), sW), x.float() @ W.float().t()),
                      (som.som_product_blocks(qd, sd, qWt.t(), sWt), dy.float() @ W.float()),
                      (som.som_product_blocks(qdt, sdt, qxt.t(), sxt), dy.float().t().contiguous() @ x.float())):
        assert float((got.float() - want).norm() / want.norm()) < 2 * 2.0 ** -4


def test_norm_to_blocks_to_product_of_one_document_and_many():
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    M, K, N = 40, 1024, 512
    h = torch.randn((M, K), generator=g, device=DEV).half()
    W = (torch.randn((N, K), generator=g, device=DEV) * K ** -0.5).half()
    qW, sW = som.som_quantise(W, 128)
    y, _, _ = som.som_rms_norm(h)
    q, s = som.som_quantise(y)
    all_rows = som.som_product_blocks(q, s, qW.t(), sW, act="gelu", dtype=torch.float16)
    for i in (0, 17, M - 1):
        q1, s1 = som.som_quantise(som.som_rms_norm(h[i:i + 1])[0])
        one = som.som_product_blocks(q1, s1, qW.t(), sW, act="gelu", dtype=torch.float16)
        # fp32 sums against the matrix instruction's, of about sqrt(K) terms of one
        assert torch.allclose(one.float(), all_rows[i:i + 1].float(), atol=2.0 ** -8, rtol=2.0 ** -9)


def test_strides_streams_graphs_and_two_workspaces():
    rng = np.random.default_rng(9)
    M, N, K = 40, 256, 4096                          # a split k axis
    x, W = _codes(M, K, 0, rng), _codes(N, K, 0, rng).t()
    xs, ws = _factors(M, K, 1, True, rng), _factors(N, K, 128, True, rng)
    assert som.som_product_blocks_workspace_bytes(M, N, K) > 0
    want = som.som_product_blocks(x, xs, W, ws)
    # one factor for all rows, one for all blocks (strides of 0)
    got = som.som_product_blocks(x, xs[:1].expand(M, K // 128), W, ws)
    assert torch.equal(got, som.som_product_blocks(x, xs[:1].repeat(M, 1), W, ws))
    got = som.som_product_blocks(x, xs, W, ws[:, :1].expand(N // 128, K // 128))
    assert torch.equal(got, som.som_product_blocks(x, xs, W, ws[:, :1].repeat(1, K // 128)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = som.som_product_blocks(x, xs, W, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    X, y = x.clone(), torch.empty_like(want)
    room = torch.empty(som.som_product_blocks_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        som.som_product_blocks(X, xs, W, ws, y=y, ws=room)
    for k in range(3):
        X.copy_(x.view(torch.uint8).roll(k, 0).view(torch.float8_e4m3fn))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, som.som_product_blocks(X, xs, W, ws))


def test_refusals_and_empty_batches():
    rng = np.random.default_rng(4)
    M, N, K = 8, 256, 300
    x, W = _codes(M, K, 0, rng), _codes(N, K, 0, rng).t()
    xs, ws = _factors(M, K, 1, True, rng), _factors(N, K, 128, True, rng)
    assert som.som_product_blocks(x[:0], xs[:0], W, ws).shape == (0, N)
    c = som.som_product_blocks
    fails = [(ValueError, lambda: c(x, xs[:7], W, ws)), (ValueError, lambda: c(x, xs[:, :2], W, ws)),
             (ValueError, lambda: c(x, xs, W, ws[:1])), (TypeError, lambda: c(x, xs.double(), W, ws)),
             (TypeError, lambda: c(x.view(torch.uint8), xs, W, ws)), (TypeError, lambda: c(x.half(), xs, W.half(), ws)),
             (ValueError, lambda: c(x, xs, W.t().contiguous().t().contiguous(), ws)), (ValueError, lambda: c(x[:, :299], xs, W, ws)),
             (ValueError, lambda: c(x, xs, W, ws, act="tanh")), (TypeError, lambda: c(x, xs, W, ws, dtype=torch.float64)),
             (TypeError, lambda: c(x, xs, W, ws, residual=torch.zeros((M, N), device=DEV))),
             (ValueError, lambda: c(x, xs, W, ws, bias=torch.zeros(N - 1, device=DEV)))]
    for error, call in fails:
        with pytest.raises(error):
            call()
