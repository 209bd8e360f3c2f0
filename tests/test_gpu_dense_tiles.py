"""The product in its large tiles (256 x 256, 256 x 128, 128 x 128; 64 x 128 in 8 bits): every
type, layout and alignment, all elements compared.  The sizes are those of `dense_plan`, whose
tiles `test_dense_plan` asserts.

Sums of small integers are exact in fp32, in the library's product that they are compared
with too.  Tolerance of the rest, u = 2^-24, t half a unit of the output type: K terms added in
any order on the matrix cores are within 2 (K + 8) u times the sum of their magnitudes; the
activation's slope is at most 1.13, and it is calculated within 2^-17 of its value; the
output is rounded once."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from dense_plan import BF16, E4M3, F16, GRADIENTS, PRODUCTS, PRODUCTS_8, tile  # noqa: E402

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"
T = {F16: torch.float16, BF16: torch.bfloat16, E4M3: torch.float8_e4m3fn}
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
U, CALC = 2.0 ** -24, 2.0 ** -17


def _inside(values, dtype, on16, fill):
    """values inside a wider array of `fill`, its rows on 16 bytes or one element off."""
    rows, cols = values.shape
    per = 16 // torch.empty((), dtype=dtype).element_size()
    lead, ld = (per, -(-cols // per) * per + 2 * per) if on16 else (1, -(-cols // per) * per + per + 3)
    wide = torch.full((rows, ld), fill, device=DEV).to(dtype)
    wide[:, lead:lead + cols] = values.to(dtype)
    view = wide[:, lead:lead + cols]
    assert (view.data_ptr() % 16 == 0 and view.stride(0) * view.element_size() % 16 == 0) == on16
    return view


def _out(rows, cols, dtype, pad=5):
    wide = torch.full((rows, cols + pad), 7.0, device=DEV).to(dtype)
    return wide, wide[:, :cols]


def _integers(g, rows, cols, most):
    return torch.randint(-most, most + 1, (rows, cols), generator=g, device=DEV).float()


def _generator(*sizes):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(s * p for s, p in zip(sizes, (17, 5, 1))))
    return g


def _same(got, want, what):
    bad = (got.double() != want.double()).nonzero()
    assert bad.numel() == 0, (what, bad.shape[0], bad[:5].tolist())


@pytest.mark.parametrize("on16", [True, False])
@pytest.mark.parametrize("elem,units", [(F16, False), (F16, True), (BF16, False), (BF16, True), (E4M3, True)])
@pytest.mark.parametrize("size", sorted(set(PRODUCTS) | set(PRODUCTS_8)))
def test_products_of_integers_are_exact(size, elem, units, on16):
    M, N, K = size
    if size not in (PRODUCTS_8 if elem == E4M3 else PRODUCTS):
        pytest.skip("this size is of the other types")
    want = PRODUCTS_8[size][0 if on16 else 1] if elem == E4M3 else PRODUCTS[size]
    assert tile(som.som.load(), M, N, K, elem, True, units, on16) == want
    g = _generator(M, N, K)
    x, W = _integers(g, M, K, 3), _integers(g, K, N, 3)
    xd = _inside(x, T[elem], on16, float("nan"))
    Wd = _inside(W.t(), T[elem], on16, float("nan")).t() if units else _inside(W, T[elem], on16, float("nan"))
    wide, y = _out(M, N, torch.float32)
    som.som_product(xd, Wd, y=y)
    _same(y, x @ W, size)
    assert bool((wide[:, N:] == 7.0).all())


@pytest.mark.parametrize("size,elem,units,on16,out", [
    ((4001, 3999, 700), BF16, False, True, torch.bfloat16), ((4001, 3999, 700), F16, True, False, torch.float32),
    ((3000, 3008, 1000), F16, False, True, torch.float16), ((4001, 3999, 700), E4M3, True, True, torch.bfloat16),
    ((2500, 2500, 520), BF16, True, True, torch.bfloat16), ((2300, 1900, 456), F16, False, False, torch.float16),
    ((2500, 2500, 900), E4M3, True, True, torch.float16), ((2048, 2048, 2000), BF16, False, True, torch.float32),
    ((1100, 2000, 333), BF16, False, False, torch.bfloat16), ((2048, 2048, 2000), E4M3, True, False, torch.float32)])
def test_epilogues(size, elem, units, on16, out):
    M, N, K = size
    g = _generator(M, N, K)
    x, W = (torch.randn(s, generator=g, device=DEV) for s in ((M, K), (K, N)))
    W *= 2 * K ** -0.5
    xd = _inside(x, T[elem], on16, float("nan"))
    Wd = _inside(W.t(), T[elem], on16, float("nan")).t() if units else _inside(W, T[elem], on16, float("nan"))
    bias = torch.randn(N, generator=g, device=DEV)
    sx = sw = None
    fx, fw = torch.ones((M, 1), device=DEV).double(), torch.ones(N, device=DEV).double()
    if elem == E4M3:
        sx, sw = (torch.rand(n, generator=g, device=DEV) + 0.5 for n in (M, N))
        fx, fw = sx.double()[:, None], sw.double()
    res = _inside(torch.randn((M, N), generator=g, device=DEV), out, False, float("nan"))
    pre_wide, pre = _out(M, N, out)
    wide, y = _out(M, N, out)
    som.som_product(xd, Wd, bias=bias, act="gelu", residual=res, alpha=-1.5, x_scale=sx, w_scale=sw, y=y, pre=pre)
    assert bool((wide[:, N:].float() == 7.0).all()) and bool((pre_wide[:, N:].float() == 7.0).all())
    x64, W64 = xd.double().contiguous(), Wd.double().contiguous()
    v = -1.5 * fx * fw * (x64 @ W64) + bias.double()
    tol = (K + 8) * 2 * U * 1.5 * fx * fw * (x64.abs() @ W64.abs()) + 4 * U * (v.abs() + bias.double().abs())
    half = HALF[out]
    assert bool(((pre.double() - v).abs() <= tol + v.abs() * half + 2.0 ** -24).all())
    a = v * 0.5 * torch.special.erfc(-v * 0.5 ** 0.5)
    want = a + res.double()
    assert bool(((y.double() - want).abs() <= 1.2 * tol + CALC * a.abs() + 4 * U * want.abs() + want.abs() * half
                 + 2.0 ** -24).all())
    again = res.clone()
    som.som_product(xd, Wd, bias=bias, act="gelu", residual=again, alpha=-1.5, x_scale=sx, w_scale=sw, y=again)
    assert torch.equal(again, y)


@pytest.mark.parametrize("on16", [True, False])
@pytest.mark.parametrize("units", [False, True])
@pytest.mark.parametrize("elem", [F16, BF16])
@pytest.mark.parametrize("size", sorted(GRADIENTS))
def test_gradients_of_integers_are_exact(size, elem, units, on16):
    M, N, K = size
    g = _generator(M, N, K)
    x, W, dy = (_integers(g, *s, 1) for s in ((M, K), (K, N), (M, N)))
    xd, dyd = (_inside(t, T[elem], on16, float("nan")) for t in (x, dy))
    Wd = _inside(W.t(), T[elem], on16, float("nan")).t() if units else _inside(W, T[elem], on16, float("nan"))
    dx, dW, dbias = som.som_product_backward(dyd, xd, Wd, alpha=2.0)
    # exact sums, rounded once
    _same(dx, (2.0 * (dy @ W.t().contiguous())).to(T[elem]), "dx")
    _same(dW, (2.0 * (x.t().contiguous() @ dy)).to(T[elem]), "dW")
    _same(dbias, dy.sum(0), "dbias")
