"""C ABI checks of the dense-document operators that need no GPU: every refusal comes
before any HIP call, workspace sizes are host-only, and empty batches of calls that
write nothing are no-ops."""

import ctypes
import os

import pytest

som = pytest.importorskip("paper_2609_05138_amd.som")

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: rejected first
ODD = ctypes.c_void_p(0x1001)
F32, F16, BF16, E4M3 = range(4)
BAD, WS = som.SOM_ERR_INVALID_ARG, som.SOM_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(som.LIB_PATH):
        pytest.fail("libsom.so is not built (run python -m paper_2609_05138_amd.build)")
    return som.load()


def _call(lib, fn, args):
    st = getattr(lib, fn)(*args.values())
    return st, lib.som_last_error().decode()


def _refuses(lib, fn, args, cases, status=BAD):
    for kw in cases:
        assert set(kw) <= set(args)
        st, msg = _call(lib, fn, dict(args, **kw))
        assert st == status and msg, (kw, st, msg)


def test_norm_refuses(lib):
    args = dict(x=FAKE, ldx=64, residual=None, ldr=0, weight=FAKE, dtype=BF16, rows=4, cols=64, eps=1e-6, q8=0, y=FAKE,
                ldy=64, h=None, ldh=0, scale=None, stream=None)
    _refuses(lib, "som_rms_norm", args, [
        dict(x=None), dict(y=None), dict(ldx=63), dict(ldy=63), dict(residual=FAKE, ldr=63), dict(h=FAKE, ldh=63),
        dict(dtype=E4M3), dict(dtype=-1), dict(dtype=4), dict(rows=-1), dict(rows=1 << 31), dict(cols=0),
        dict(cols=1 << 31, ldx=1 << 31, ldy=1 << 31), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
        dict(q8=2), dict(q8=1), dict(scale=FAKE), dict(x=ODD), dict(y=ODD), dict(weight=ODD), dict(residual=ODD, ldr=64),
        dict(h=ODD, ldh=64), dict(q8=1, scale=ODD), dict(ldx=1 << 41), dict(rows=1 << 30, ldx=1 << 40),
        dict(dtype=F32, x=ctypes.c_void_p(0x1002))])
    assert _call(lib, "som_rms_norm", dict(args, rows=0, x=None, y=None)) == (som.SOM_OK, "")


def test_norm_gradient_refuses(lib):
    args = dict(dy=FAKE, lddy=64, h=FAKE, ldh=64, weight=None, dh=None, lddh=0, dtype=F16, rows=4, cols=64, eps=1e-6,
                dx=FAKE, lddx=64, dweight=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)
    _refuses(lib, "som_rms_norm_backward", args, [
        dict(dy=None), dict(h=None), dict(dx=None), dict(lddy=1), dict(ldh=1), dict(lddx=1), dict(dh=FAKE, lddh=63),
        dict(dtype=E4M3), dict(rows=-1), dict(cols=0), dict(eps=-0.5), dict(dweight=ODD), dict(dy=ODD), dict(h=ODD),
        dict(dx=ODD), dict(weight=ODD), dict(ws=ctypes.c_void_p(0x1010))])
    _refuses(lib, "som_rms_norm_backward", args, [dict(ws=None), dict(ws_bytes=16)], WS)
    assert _call(lib, "som_rms_norm_backward", dict(args, rows=0, dweight=None, ws=None))[0] == som.SOM_OK
    size = lib.som_rms_norm_backward_workspace_bytes
    assert size(0, 64) == 0 and size(4, 0) == 0 and size(-1, 64) == 0 and size(1 << 31, 64) == 0
    for rows, cols in ((1, 1), (8192, 4096), (3, 100000)):
        assert size(rows, cols) >= 4 * cols and size(rows, cols) % 256 == 0


def _epilogue(**kw):
    e = som.som_epilogue(alpha=1.0)
    for k, v in kw.items():
        setattr(e, k, v)
    return ctypes.byref(e)


def test_product_refuses(lib):
    args = dict(x=FAKE, ldx=64, W=FAKE, ldw=32, w_units=0, x_dtype=BF16, M=4, N=32, K=64, y=FAKE, ldy=32, y_dtype=BF16,
                e=None, ws=FAKE, ws_bytes=1 << 30, stream=None)
    _refuses(lib, "som_product", args, [
        dict(x=None), dict(W=None), dict(y=None), dict(ldx=63), dict(ldw=31), dict(ldy=31), dict(w_units=1), dict(w_units=2),
        dict(w_units=-1, ldw=64), dict(x_dtype=F32), dict(x_dtype=4), dict(x_dtype=E4M3), dict(y_dtype=F16),
        dict(y_dtype=E4M3), dict(x_dtype=E4M3, w_units=1, ldw=64, y_dtype=E4M3), dict(M=-1), dict(N=0), dict(K=0),
        dict(M=1 << 31), dict(N=(1 << 30) + 1, ldw=1 << 31, ldy=1 << 31), dict(K=(1 << 30) + 1, ldx=1 << 31),
        dict(M=1 << 30, N=1 << 30, ldw=1 << 30, ldy=1 << 30), dict(x=ODD), dict(W=ODD), dict(y=ODD),
        dict(e=_epilogue(act=5)), dict(e=_epilogue(act=-1)), dict(e=_epilogue(reserved=1)),
        dict(e=_epilogue(residual=0x1000, ldr=31)), dict(e=_epilogue(residual=0x1001, ldr=32)),
        dict(e=_epilogue(pre=0x1000, ldp=31)), dict(e=_epilogue(bias=0x1002)), dict(e=_epilogue(x_scale=0x1001)),
        dict(e=_epilogue(w_scale=0x1003))])
    assert _call(lib, "som_product", dict(args, M=0, x=None, y=None))[0] == som.SOM_OK
    # few rows and a long k axis: the axis is split, and the parts need room
    need = lib.som_product_workspace_bytes(4, 32, 1 << 14, BF16)
    assert need > 0 and need % 256 == 0
    long = dict(args, K=1 << 14, ldx=1 << 14)
    _refuses(lib, "som_product", long, [dict(ws=None), dict(ws_bytes=need - 1)], WS)
    _refuses(lib, "som_product", long, [dict(ws=ctypes.c_void_p(0x1010))])
    size = lib.som_product_workspace_bytes
    assert size(0, 1, 1, BF16) == 0 and size(1, 0, 1, BF16) == 0 and size(1, 1, 0, BF16) == 0 and size(9, 9, 9, F32) == 0


def test_product_refuses_more_than_a_launch_holds(lib):
    # ceil(M / 256) ceil(N / 128) up to 2^23 - 8
    args = dict(x=FAKE, ldx=64, W=FAKE, ldw=1 << 30, w_units=0, x_dtype=BF16, M=4, N=32, K=64, y=FAKE, ldy=1 << 30,
                y_dtype=BF16, e=None, ws=None, ws_bytes=0, stream=None)
    _refuses(lib, "som_product", args, [dict(M=1, N=1 << 30), dict(M=(1 << 31) - 1, N=128, ldy=128),
                                        dict(M=1 << 20, N=1 << 19)])


def test_product_gradient_refuses(lib):
    args = dict(dy=FAKE, lddy=32, x=FAKE, ldx=64, W=FAKE, ldw=32, w_units=0, dtype=F16, M=4, N=32, K=64, act=4, pre=FAKE,
                ldp=32, alpha=1.0, dx=FAKE, lddx=64, dW=FAKE, lddw=32, dbias=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)
    _refuses(lib, "som_product_backward", args, [
        dict(dy=None), dict(x=None), dict(W=None), dict(pre=None), dict(lddy=31), dict(ldx=63), dict(ldw=31), dict(ldp=31),
        dict(lddx=63), dict(lddw=31), dict(w_units=1), dict(w_units=3), dict(dtype=F32), dict(dtype=E4M3), dict(act=5),
        dict(M=-1), dict(N=0), dict(K=0), dict(dbias=ODD), dict(dy=ODD), dict(dx=ODD), dict(dW=ODD), dict(pre=ODD),
        dict(ws=ctypes.c_void_p(0x1010))])
    _refuses(lib, "som_product_backward", args, [dict(ws=None), dict(ws_bytes=16)], WS)
    nothing = dict(args, M=0, dW=None, dbias=None)
    assert _call(lib, "som_product_backward", nothing)[0] == som.SOM_OK
    size = lib.som_product_backward_workspace_bytes
    assert size(0, 8, 8, F16) == 0 and size(8, 8, 8, E4M3) == 0
    assert size(1000, 777, 500, BF16) >= 2 * 1000 * 777


def test_dropout_refuses(lib):
    args = dict(x=FAKE, ldx=64, residual=None, ldr=0, dtype=BF16, rows=4, cols=64, p=0.1, seed=1, offset=0, y=FAKE, ldy=64,
                stream=None)
    _refuses(lib, "som_dropout", args, [
        dict(x=None), dict(y=None), dict(ldx=63), dict(ldy=63), dict(residual=FAKE, ldr=63), dict(dtype=E4M3),
        dict(rows=-1), dict(rows=1 << 32), dict(cols=0), dict(cols=1 << 31), dict(p=-0.1), dict(p=1.1),
        dict(p=float("nan")), dict(x=ODD), dict(y=ODD), dict(residual=ODD, ldr=64)])
    assert _call(lib, "som_dropout", dict(args, rows=0, x=None, y=None))[0] == som.SOM_OK


def test_the_binding_refuses_cpu_tensors(lib):
    import torch
    x, W = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((8, 8), dtype=torch.bfloat16)
    for call in (lambda: som.som_rms_norm(x), lambda: som.som_rms_norm_backward(x, x), lambda: som.som_product(x, W),
                 lambda: som.som_product_backward(x, x, W), lambda: som.som_dropout(x, 0.5, 1)):
        with pytest.raises(ValueError):
            call()
