"""The norm of rows that are not finite, too long for fp32's sum of squares, or zero: what the
header says of them, in every kernel form, and that the rows beside them are not touched."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [40, 1000, 2050, 4096, 9000, 40000])
def test_rows_of_the_header(cols, kind):
    x = torch.randn((7, cols), device=DEV).to(kind)
    x[1, cols // 3] = float("nan")
    x[2, cols - 1] = float("-inf")
    x[3] = 1e30                          # finite; its squares are not
    x[4] = 0.0
    plain = som.som_rms_norm(x[:1].clone(), None, 1e-6)[0]
    for eps in (1e-6, 0.0):
        y, _, _ = som.som_rms_norm(x, None, eps)
        q, _, scale = som.som_rms_norm(x, None, eps, q8=True)
        q = q.float()
        assert bool(y[1].isnan().all()) and bool(q[1].isnan().all()) and bool(scale[1].isnan())
        assert bool(y[2, -1].isnan()) and bool((y[2, :-1] == 0).all())
        assert bool(q[2].isnan().all()) and bool(scale[2].isnan())
        assert bool((y[3] == 0).all()) and bool((q[3] == 0).all()) and float(scale[3]) == 1.0
        if eps:
            assert bool((y[4] == 0).all()) and bool((q[4] == 0).all()) and float(scale[4]) == 1.0
            assert torch.equal(y[:1], plain)
        else:
            assert bool(y[4].isnan().all()) and bool(q[4].isnan().all()) and bool(scale[4].isnan())
        for i in (0, 5, 6):
            assert bool(y[i].isfinite().all()) and float(q[i].abs().max()) == 448.0
            assert bool(scale[i].isfinite())


@pytest.mark.parametrize("cols", [40, 1000, 2050, 4096, 9000, 20000])
def test_the_gradient_of_rows_beside_them(cols):
    h, dy = (torch.randn((9, cols), device=DEV) for _ in range(2))
    want, _ = som.som_rms_norm_backward(dy, h, None, 1e-6)
    h[1, 0], h[4, cols - 1], h[7] = float("nan"), float("inf"), 1e30
    dx, dweight = som.som_rms_norm_backward(dy, h, None, 1e-6)
    keep = [0, 2, 3, 5, 6, 8]
    assert torch.equal(dx[keep], want[keep])
    # the columns of the NaN and the infinity; a NaN's row has no s at all
    assert bool(dweight.isnan().all())


@pytest.mark.parametrize("rows", [1, 4, 16, 256])
def test_every_code_of_8_bits(rows):
    codes = torch.arange(256, dtype=torch.uint8, device=DEV)
    values = codes.view(torch.float8_e4m3fn).float()         # +-0, subnormal and normal values, two NaNs
    x = torch.zeros((256, 48), dtype=torch.uint8, device=DEV)
    x[:, 33] = codes
    x = x.view(torch.float8_e4m3fn)
    W = torch.zeros((20, 48), device=DEV)
    W[:, 33] = 1.0
    W = W.to(torch.float8_e4m3fn).t()
    got = torch.cat([som.som_product(x[a:a + rows], W, dtype=torch.float32) for a in range(0, 256, rows)])
    want = values[:, None].expand(256, 20)
    assert int(values.isnan().sum()) == 2
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
