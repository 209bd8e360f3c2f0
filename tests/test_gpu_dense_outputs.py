"""Gradients of which only some are wanted: each is the same, bit for bit, as when all are
asked for, and the inputs that only an unwanted one reads may be absent at the C entry."""

import ctypes
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"


def _inputs(M, N, K, kind, units):
    x, dy, pre = (torch.randn(s, device=DEV).to(kind) for s in ((M, K), (M, N), (M, N)))
    W = (torch.randn((K, N), device=DEV) * K ** -0.5).to(kind)
    return x, W.t().contiguous().t() if units else W, dy, pre


@pytest.mark.parametrize("units", [False, True])
@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("M,N,K", [(1, 40, 24), (300, 136, 129), (700, 520, 1000)])
def test_some_gradients_of_a_product(M, N, K, act, kind, units):
    x, W, dy, pre = _inputs(M, N, K, kind, units)
    all_of = som.som_product_backward(dy, x, W, act=act, pre=pre, alpha=0.5)
    for need in itertools.product((False, True), repeat=3):
        got = som.som_product_backward(dy, x, W, act=act, pre=pre, alpha=0.5, need_dx=need[0], need_dW=need[1],
                                       need_dbias=need[2])
        for g, a, n in zip(got, all_of, need):
            assert torch.equal(g, a) if n else g is None, need


def test_an_unwanted_gradient_has_no_place():
    x, W, dy, pre = _inputs(8, 16, 8, torch.float16, False)
    with pytest.raises(ValueError):
        som.som_product_backward(dy, x, W, dx=torch.empty_like(x), need_dx=False)
    with pytest.raises(ValueError):
        som.som_rms_norm_backward(x, x, dweight=torch.empty(8, device=DEV), need_dweight=False)


@pytest.mark.parametrize("rows,cols", [(1, 7), (300, 512), (9, 2048), (600, 4096), (70, 20000)])
def test_a_norms_gradient_without_the_weights(rows, cols):
    h, dy = (torch.randn((rows, cols), device=DEV).to(torch.bfloat16) for _ in range(2))
    w = torch.randn(cols, device=DEV).to(torch.bfloat16)
    want, _ = som.som_rms_norm_backward(dy, h, w)
    dx, dweight = som.som_rms_norm_backward(dy, h, w, need_dweight=False)
    assert dweight is None and torch.equal(dx, want)


@pytest.mark.parametrize("units", [0, 1])
@pytest.mark.parametrize("act", [0, 4])
def test_inputs_of_unwanted_gradients_may_be_absent(act, units):
    M, N, K = 130, 72, 200
    x, W, dy, pre = _inputs(M, N, K, torch.bfloat16, bool(units))
    want = som.som_product_backward(dy, x, W, act="silu" if act else "none", pre=pre)
    lib = som.som.load()
    ws = torch.empty(lib.som_product_backward_workspace_bytes(M, N, K, 2), dtype=torch.uint8, device=DEV)
    ldw = K if units else N
    p = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())
    for need in itertools.product((False, True), repeat=3):
        dx, dbias = torch.full_like(want[0], 9.0), torch.full_like(want[2], 9.0)
        dW = torch.full((N, K) if units else (K, N), 9.0, dtype=torch.bfloat16, device=DEV)
        status = lib.som_product_backward(
            p(dy), N, p(x) if need[1] else None, K, p(W) if need[0] else None, ldw, units, 2, M, N, K, act,
            p(pre) if act else None, N, 1.0, p(dx) if need[0] else None, K, p(dW) if need[1] else None, ldw,
            p(dbias) if need[2] else None, p(ws), ws.numel(), torch.cuda.current_stream().cuda_stream)
        assert status == 0, lib.som_last_error()
        got = (dx, dW.t() if units else dW, dbias)
        for g, a, n in zip(got, want, need):
            assert torch.equal(g, a) if n else bool((g == 9.0).all()), need
