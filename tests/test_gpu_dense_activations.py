"""The activations and their derivatives alone, in fp32, over the range where they are not
yet constant.  The argument is exact (a bias of fp32 values on a product of zeros; for the
gradient a 16-bit argument, and dbias of one row, which is not rounded).

Relative bounds, r (u = 2^-24): the hardware's exponential and reciprocal are within 2 u
each; an exponent's argument a, of `n` roundings, costs n u |a| of the exponential.
  silu       s = 1 / (1 + e^-v): a = -v, n = 2
  gelu_tanh  s of k (v + c v^3), n = 5
  gelu       the normal distribution's share below v: its rational form within 2^-19, and
             e^(-v^2 / 2), n = 3
A factor of two is left on each.  Differences of the derivative's terms are bounded by the
terms' magnitudes."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"
U = 2.0 ** -24
K, C = 2.0 * math.sqrt(2.0 / math.pi), 0.044715
# beyond, results are below fp32's normal numbers or the argument itself
RANGE = {"relu": 1e30, "gelu": 10.0, "gelu_tanh": 8.0, "silu": 80.0}
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def _value(act, v):
    """(value, relative bound)."""
    if act == "relu":
        return np.maximum(v, 0.0), 0.0 * v
    if act == "gelu":
        return 0.5 * v * _erfc(-v / math.sqrt(2.0)), 2 * (2.0 ** -19 + 8 * U + 3 * U * 0.5 * v * v)
    z, n = (v, 2) if act == "silu" else (K * (v + C * v ** 3), 5)
    return v * _sigmoid(z), 2 * (8 * U + n * U * np.abs(z))


def _slope(act, v):
    """(derivative, absolute bound)."""
    if act == "relu":
        return (v > 0).astype(np.float64), 0.0 * v
    if act == "gelu":
        below, bell = 0.5 * _erfc(-v / math.sqrt(2.0)), v * np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
        r = _value(act, v)[1]
        return below + bell, r * (below + np.abs(bell))
    z, dz = (v, np.ones_like(v)) if act == "silu" else (K * (v + C * v ** 3), K * (1.0 + 3.0 * C * v * v))
    s, r = _sigmoid(z), _value(act, v)[1]
    # s + v s (1 - s) dz: 1 - s is off by what s is
    return s + v * s * (1.0 - s) * dz, r * s * (1.0 + np.abs(v) * dz * (1.0 - s)) + s * np.abs(v) * dz * (r * s + U)


def _arguments(act):
    top = RANGE[act]
    near = np.linspace(-min(top, 4.0), min(top, 4.0), 6001)
    return np.concatenate([np.linspace(-top, top, 12001), near, [0.0, 1e-30, -1e-30]])


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_values(act, rows):
    v = torch.as_tensor(_arguments(act)).float()
    x = torch.zeros((rows, 16), dtype=torch.float16, device=DEV)
    W = torch.zeros((16, v.numel()), dtype=torch.float16, device=DEV)
    y = som.som_product(x, W, bias=v.to(DEV), act=act, dtype=torch.float32).double().cpu().numpy()
    want, r = _value(act, v.double().numpy())
    bad = ~(np.abs(y - want) <= r * np.abs(want) + 2.0 ** -126)
    assert not bad.any(), (int(bad.sum()), v.numpy()[bad[0]][:5], y[0][bad[0]][:5], want[bad[0]][:5])


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_derivatives(act, kind):
    pre = torch.as_tensor(np.clip(_arguments(act), -6e4, 6e4)).to(kind)
    v = pre.double().numpy()
    pre = pre.to(DEV)[None]
    x, W = torch.ones((1, 8), dtype=kind, device=DEV), torch.zeros((8, v.size), dtype=kind, device=DEV)
    _, _, dbias = som.som_product_backward(torch.ones_like(pre), x, W, act=act, pre=pre)
    got = dbias.double().cpu().numpy()
    want, tol = _slope(act, v)
    bad = ~(np.abs(got - want) <= tol + 2.0 ** -126)
    assert not bad.any(), (int(bad.sum()), v[bad][:5], got[bad][:5], want[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("rows", [1, 40])
def test_gelu_of_what_is_not_finite(rows):
    v = torch.tensor([float("inf"), 3e38, 1e20, 20.0, 0.0, -20.0, -1e20, -3e38, float("-inf"), float("nan")])
    x = torch.zeros((rows, 16), dtype=torch.float16, device=DEV)
    W = torch.zeros((16, v.numel()), dtype=torch.float16, device=DEV)
    y = som.som_product(x, W, bias=v.to(DEV), act="gelu", dtype=torch.float32).cpu()
    assert bool(y[:, 9].isnan().all())
    want = torch.where(v > 0, v, torch.zeros_like(v))[:9]      # the limit
    assert torch.equal(y[:, :9], want.expand(rows, 9))
