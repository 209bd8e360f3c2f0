"""The binding of what trains and serves the dense layer with more than one device, without a GPU:
tensors that say which device they are on, and a library that notes the current one."""

import pytest

torch = pytest.importorskip("torch")
som = pytest.importorskip("paper_2609_05138_amd.som")

from test_dense_devices import _on, _Stream, world  # noqa: E402,F401

BF, Q8, I32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32


def _calls(a, b, stream=None):
    """Every operator, its first tensor on device a, another one on device b."""
    m = lambda i, *s: _on(i, torch.zeros(s, dtype=BF))
    f = lambda i, *s: _on(i, torch.zeros(s))
    q = lambda i, *s: _on(i, torch.zeros(s).to(Q8))
    n = lambda i: _on(i, torch.zeros(4, dtype=I32))
    ws = lambda i: _on(i, torch.zeros(512, dtype=torch.uint8))
    k = dict(stream=stream)
    loss = lambda **o: som.som_cross_entropy(m(a, 4, 8), o.pop("W", m(a, 8, 6)), o.pop("labels", n(a)),
                                             **{"loss": f(a, 4), "lse": f(a, 4), **o}, **k)
    back = lambda **o: som.som_cross_entropy_backward(
        o.pop("dloss", f(a, 4)), m(a, 4, 8), o.pop("W", m(a, 8, 6)), o.pop("labels", n(a)), o.pop("lse", f(a, 4)),
        **{"dx": m(a, 4, 8), "dW": m(a, 8, 6), "dbias": f(a, 6), **o}, **k)
    quant = lambda **o: som.som_quantise(m(a, 4, 200), **{"q": q(a, 4, 200), "scale": f(a, 4, 2), **o}, **k)
    blocks = lambda **o: som.som_product_blocks(
        q(a, 4, 200), o.pop("xs", f(a, 4, 2)), o.pop("W", q(a, 6, 200)).t(), o.pop("ws_", f(a, 1, 2)),
        **{"y": m(a, 4, 6), **o}, **k)
    ortho = lambda **o: som.som_orthogonalise(m(a, 4, 8), **{"y": m(a, 4, 8), **o}, **k)
    return {
        "loss": [lambda: loss(W=m(b, 8, 6)), lambda: loss(W=m(b, 6, 8).t()), lambda: loss(labels=n(b)),
                 lambda: loss(bias=f(b, 6)), lambda: loss(loss=f(b, 4)), lambda: loss(lse=f(b, 4)), lambda: loss(ws=ws(b))],
        "loss's gradient": [lambda: back(dloss=f(b, 4)), lambda: back(W=m(b, 8, 6)), lambda: back(labels=n(b)),
                            lambda: back(lse=f(b, 4)), lambda: back(bias=f(b, 6)), lambda: back(dx=m(b, 4, 8)),
                            lambda: back(dW=m(b, 8, 6)), lambda: back(dbias=f(b, 6)), lambda: back(ws=ws(b))],
        "quantise": [lambda: quant(q=q(b, 4, 200)), lambda: quant(scale=f(b, 4, 2))],
        "blocks": [lambda: blocks(xs=f(b, 4, 2)), lambda: blocks(W=q(b, 6, 200)), lambda: blocks(ws_=f(b, 1, 2)),
                   lambda: blocks(bias=f(b, 6)), lambda: blocks(residual=m(b, 4, 6)), lambda: blocks(y=m(b, 4, 6)),
                   lambda: blocks(pre=m(b, 4, 6)), lambda: blocks(ws=ws(b))],
        "orthogonalise": [lambda: ortho(y=m(b, 4, 8)), lambda: ortho(ws=ws(b))],
    }


def test_tensors_of_one_call_are_on_one_device(world):  # noqa: F811
    for name, calls in _calls(0, 1).items():
        for i, call in enumerate(calls):
            with pytest.raises(ValueError, match="cuda:"):
                call()
            assert not world["calls"], (name, i)


@pytest.mark.parametrize("index", [0, 1])
def test_a_call_runs_on_its_tensors_device(world, index):  # noqa: F811
    for name, calls in _calls(index, index).items():
        for call in calls:
            world["calls"].clear()
            call()
            (_, current, stream), = world["calls"]
            assert current == index and stream == 500 + index, name
    assert world["current"] == 0


def test_a_stream_of_another_device_is_refused(world):  # noqa: F811
    for calls in _calls(1, 1, _Stream(0)).values():
        with pytest.raises(ValueError, match="stream"):
            calls[0]()
    assert not world["calls"]
    for calls in _calls(1, 1, _Stream(1)).values():
        world["calls"].clear()
        calls[0]()
        assert [(c[1], c[2]) for c in world["calls"]] == [(1, 1001)]
