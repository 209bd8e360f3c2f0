"""The dense binding with more than one device, without a GPU: tensors that say which device
they are on, and a library that notes the current one."""

import contextlib

import pytest

torch = pytest.importorskip("torch")
som = pytest.importorskip("paper_2609_05138_amd.som")


class _On(torch.Tensor):
    """A tensor that says it is on cuda:<index>."""

    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index

    def t(self):
        return _on(self.index, super().t())


def _on(index, t):
    t = t.as_subclass(_On)
    t.index = index
    return t


class _Stream:
    def __init__(self, index):
        self.device_index, self.device, self.cuda_stream = index, torch.device("cuda", index), 1000 + index


class _Library:
    """Every entry point notes the current device and the stream, and succeeds."""

    def __init__(self, world):
        self.world = world

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 0
        return lambda *a: self.world["calls"].append((name, self.world["current"], a[-1])) or 0


@pytest.fixture
def world(monkeypatch):
    w = {"current": 0, "calls": []}

    @contextlib.contextmanager
    def device(d):
        before, w["current"] = w["current"], torch.device(d).index if not isinstance(d, int) else d
        yield
        w["current"] = before

    monkeypatch.setattr(som, "load", lambda: _Library(w))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: w["current"], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 500 + d, raising=False)
    return w


BF = torch.bfloat16


def _calls(a, b, stream=None):
    """Every operator, its first tensor on device a, another one on device b."""
    m = lambda i, *s: _on(i, torch.zeros(s, dtype=BF))
    f = lambda i, n: _on(i, torch.zeros(n))
    k = dict(stream=stream)
    norm = lambda **o: som.som_rms_norm(m(a, 4, 8), **{"y": m(a, 4, 8), **o}, **k)
    back = lambda **o: som.som_rms_norm_backward(o.pop("dy", m(a, 4, 8)), m(a, 4, 8),
                                                 **{"dx": m(a, 4, 8), "dweight": f(a, 8), **o}, **k)
    product = lambda W=None, **o: som.som_product(m(a, 4, 8), m(a, 8, 8) if W is None else W,
                                                  **{"y": m(a, 4, 8), **o}, **k)
    pback = lambda **o: som.som_product_backward(
        o.pop("dy", m(a, 4, 8)), m(a, 4, 8), o.pop("W", m(a, 8, 8)),
        **{"dx": m(a, 4, 8), "dW": m(a, 8, 8), "dbias": f(a, 8), **o}, **k)
    drop = lambda **o: som.som_dropout(m(a, 4, 8), 0.5, 1, **{"y": m(a, 4, 8), **o}, **k)
    ws = lambda i: _on(i, torch.zeros(512, dtype=torch.uint8))
    return {
        "norm": [lambda: norm(weight=_on(b, torch.zeros(8, dtype=BF))), lambda: norm(y=m(b, 4, 8)),
                 lambda: norm(residual=m(b, 4, 8), h=m(a, 4, 8)), lambda: norm(residual=m(a, 4, 8), h=m(b, 4, 8)),
                 lambda: norm(q8=True, y=_on(a, torch.zeros((4, 8)).to(torch.float8_e4m3fn)), scale=f(b, 4))],
        "norm's gradient": [lambda: back(dy=m(b, 4, 8)), lambda: back(dh=m(b, 4, 8)), lambda: back(dx=m(b, 4, 8)),
                            lambda: back(dweight=f(b, 8)), lambda: back(ws=ws(b))],
        "product": [lambda: product(m(b, 8, 8)), lambda: product(m(b, 8, 8).t()), lambda: product(bias=f(b, 8)),
                    lambda: product(residual=m(b, 4, 8)), lambda: product(y=m(b, 4, 8)),
                    lambda: product(pre=m(b, 4, 8)),
                    lambda: product(x_scale=f(b, 4)), lambda: product(w_scale=f(b, 8)), lambda: product(ws=ws(b))],
        "product's gradient": [lambda: pback(dy=m(b, 4, 8)), lambda: pback(W=m(b, 8, 8)), lambda: pback(dx=m(b, 4, 8)),
                               lambda: pback(dW=m(b, 8, 8)), lambda: pback(dbias=f(b, 8)),
                               lambda: pback(act="silu", pre=m(b, 4, 8)), lambda: pback(ws=ws(b))],
        "dropout": [lambda: drop(y=m(b, 4, 8)), lambda: drop(residual=m(b, 4, 8))],
    }


def test_tensors_of_one_call_are_on_one_device(world):
    for name, calls in _calls(0, 1).items():
        for i, call in enumerate(calls):
            with pytest.raises(ValueError, match="cuda:"):
                call()
            assert not world["calls"], (name, i)


@pytest.mark.parametrize("index", [0, 1])
def test_a_call_runs_on_its_tensors_device(world, index):
    for name, calls in _calls(index, index).items():
        for call in calls:
            world["calls"].clear()
            call()
            (_, current, stream), = world["calls"]
            assert current == index and stream == 500 + index, name
    assert world["current"] == 0


def test_a_stream_of_another_device_is_refused(world):
    for calls in _calls(1, 1, _Stream(0)).values():
        with pytest.raises(ValueError, match="stream"):
            calls[0]()
    assert not world["calls"]
    for calls in _calls(1, 1, _Stream(1)).values():
        world["calls"].clear()
        calls[0]()
        assert [(c[1], c[2]) for c in world["calls"]] == [(1, 1001)]
