"""The norm's gradient with eps = 0, at row counts that leave a workgroup's last rows
empty (eight rows share one up to 512 columns, two up to 2,048)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import dense as oracle  # noqa: E402

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}
U, CALC = 2.0 ** -24, 2.0 ** -17


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 512), (7, 300), (8, 512), (9, 512), (3, 2048), (4, 513), (4097, 512),
                                       (1025, 2047), (3, 4096), (2, 20000)])
def test_norm_gradient_without_eps(rows, cols, kind):
    rng = np.random.default_rng(rows * 131 + cols)
    # no row is zero: the formula is finite with eps = 0
    h, dy, dh = (torch.as_tensor(rng.normal(size=(rows, cols)) * s).to(DEV).to(T[kind]) for s in (2.0, 0.3, 0.2))
    h[:, 0] = 1.0
    w = torch.as_tensor(rng.normal(1.0, 0.2, cols)).to(DEV).to(T[kind])
    h64, dy64, dh64, w64 = (t.double().cpu().numpy() for t in (h, dy, dh, w))
    for weight, extra in ((w, dh), (None, None)):
        g = dy64 * w64 if weight is not None else dy64
        want, dw = oracle.rms_norm_backward(dy64, h64, None if weight is None else w64, 0.0,
                                            None if extra is None else dh64)
        dx, dweight = som.som_rms_norm_backward(dy, h, weight, 0.0, dh=extra)
        # a row's sums have `cols` terms, added at most cols / 64 + 64 deep; the columns' `rows`
        s = 1.0 / np.sqrt((h64 ** 2).mean(1, keepdims=True))
        calc = CALC + (cols / 64 + 64) * U
        size = np.abs(s * g) + np.abs(h64) * s ** 3 * np.abs(g * h64).mean(1, keepdims=True)
        size = size + (0 if extra is None else np.abs(dh64))
        got, gw = dx.double().cpu().numpy(), dweight.double().cpu().numpy()
        assert (np.abs(gw - dw) <= np.abs(dy64 * h64 * s).sum(0) * (2 * calc + rows * U) + 1e-30).all()
        assert (np.abs(got - want) <= np.abs(want) * HALF[kind] + size * 2 * calc + TINY[kind]).all()
