"""What trains and serves the dense layer, together: the example with its given units, orthogonalised
updates and blocks of 8 bits, its loss's gradient, and a whole step captured into a graph."""

import importlib.util
import math
import os

import numpy as np
import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import train as oracle  # noqa: E402

if torch.cuda.is_available():
    import paper_2609_05138_amd as som
else:  # collected on CPU-only machines, never run there
    som = None

DEV = "cuda:0"


def _example():
    spec = importlib.util.spec_from_file_location("dense_map", os.path.join(ROOT, "examples", "dense_map.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("given,orthogonal,blocks", [(True, True, True), (True, False, False), (False, True, False),
                                                     (False, False, True)])
def test_the_example_runs(given, orthogonal, blocks):
    lines = []
    losses, same = _example().main(steps=3, docs=150, states=200, side=9, features=75, say=lines.append, given=given,
                                   orthogonal=orthogonal, blocks=blocks)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses) and lines and 0.0 <= same <= 1.0


def test_the_examples_gradient_against_differences():
    rng = np.random.default_rng(0)
    docs, features, N = 9, 24, 30
    codebook = torch.as_tensor(rng.uniform(size=(features, 32)), device=DEV).half()
    norms = som.som_codebook_norms(codebook, N=N)
    z = torch.as_tensor(rng.uniform(size=(docs, features)), device=DEV).half()
    units = torch.as_tensor(rng.integers(0, N, docs), dtype=torch.int32, device=DEV)
    t, scale = 2.0, float(docs)
    loss, dz = _example().given_loss(z, codebook, N, norms, units, t, scale)
    w, zn, u = codebook[:, :N].double().cpu().numpy(), z.double().cpu().numpy(), units.cpu().numpy()

    def f(a):
        d = -t * ((a[:, :, None] - w[None]) ** 2).sum(1)
        return float((np.log(np.exp(d).sum(1)) - d[np.arange(docs), u]).mean())

    assert abs(float(loss) - f(zn)) < 1e-5
    h = 1e-5
    for at in [(0, 0), (3, 7), (8, 23), (5, 11)]:
        up, down = zn.copy(), zn.copy()
        up[at] += h
        down[at] -= h
        want = scale * (f(up) - f(down)) / (2 * h)
        # g and dz in fp16: half a step each of sums of terms of up to 2 t
        assert abs(float(dz[at]) - want) <= 2.0 ** -10 * (abs(want) + 2 * t)


def _step(x, r, gain, W, bias, label, out, ws):
    """norm -> product -> scores' loss -> gradients -> orthogonalised update, in the given buffers."""
    som.som_rms_norm(x, gain, residual=r, y=out["y"], h=out["h"])
    som.som_product(out["y"], W, bias=bias, act="silu", pre=out["pre"], y=out["z"], ws=ws[0])
    som.som_cross_entropy(out["z"], out["units"], label, loss=out["loss"], lse=out["lse"], ws=ws[1])
    som.som_cross_entropy_backward(out["dloss"], out["z"], out["units"], label, out["lse"], dx=out["dz"],
                                   dW=out["dunits"], dbias=out["dub"], ws=ws[2])
    som.som_product_backward(out["dz"], out["y"], W, act="silu", pre=out["pre"], dx=out["dy"], dW=out["dW"],
                             dbias=out["db"], ws=ws[3])
    som.som_orthogonalise(out["dW"], y=out["step"], ws=ws[4])
    som.som_quantise(out["z"], q=out["q"], scale=out["s"])
    som.som_product_blocks(out["q"], out["s"], out["q8"].t(), out["s8"], y=out["served"], ws=ws[5])


def test_a_whole_step_captured_and_replayed():
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    M, K, F, N = 120, 200, 264, 500
    bf = torch.bfloat16
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x, r = rnd(M, K).to(bf), rnd(M, K).to(bf)
    gain, W, bias = torch.ones(K, device=DEV).to(bf), (rnd(K, F) * K ** -0.5).to(bf), 0.1 * rnd(F)
    units = (rnd(N, F) * F ** -0.5).to(bf)
    label = torch.randint(-1, N, (M,), generator=g, device=DEV).int()
    q8, s8 = som.som_quantise(units, 128)
    e = lambda *s: torch.empty(s, dtype=bf, device=DEV)  # noqa: E731

    def buffers():
        return dict(y=e(M, K), h=e(M, K), pre=e(M, F), z=e(M, F), units=units.t(), loss=torch.empty(M, device=DEV),
                    lse=torch.empty(M, device=DEV), dloss=torch.full((M,), 1.0 / M, device=DEV), dz=e(M, F),
                    dunits=e(N, F).t(), dub=torch.empty(N, device=DEV), dy=e(M, K), dW=e(K, F), db=torch.empty(F, device=DEV),
                    step=e(K, F), q=torch.empty((M, F), dtype=torch.float8_e4m3fn, device=DEV),
                    s=torch.empty((3, M), device=DEV).t(), q8=q8, s8=s8, served=e(M, N))

    def rooms():
        sizes = (som.som_product_workspace_bytes(M, F, K), som.som_cross_entropy_workspace_bytes(M, N, F),
                 som.som_cross_entropy_backward_workspace_bytes(M, N, F), som.som_product_backward_workspace_bytes(M, F, K),
                 som.som_orthogonalise_workspace_bytes(K, F), som.som_product_blocks_workspace_bytes(M, N, F))
        return [torch.empty(max(n, 256), dtype=torch.uint8, device=DEV) for n in sizes]

    out, ws = buffers(), rooms()
    X, L = x.clone(), label.clone()
    _step(X, r, gain, W, bias, L, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(X, r, gain, W, bias, L, out, ws)
    eager, room = buffers(), rooms()
    for k in range(3):
        X.copy_(x * (1.0 + 0.5 * k))
        L.copy_(label.roll(k))
        graph.replay()
        torch.cuda.synchronize()
        _step(X, r, gain, W, bias, L, eager, room)
        for name in out:
            a, b = out[name].contiguous(), eager[name].contiguous()
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (k, name)
    # and against the formulas, from the rounded values that each operator was given
    f64 = lambda v: v.double().cpu().numpy()  # noqa: E731
    want, _ = oracle.cross_entropy(f64(out["z"]), f64(units).T, L.cpu().numpy().astype(np.int64))
    assert np.abs(f64(out["loss"]) - want).max() < 1e-4
    dz, dunits, dub, _ = oracle.cross_entropy_backward(f64(out["dloss"]), f64(out["z"]), f64(units).T,
                                                       L.cpu().numpy().astype(np.int64))
    for got, exact, tol in ((out["dz"], dz, 2.0 ** -7), (out["dunits"], dunits, 2.0 ** -7), (out["dub"], dub, 2.0 ** -16)):
        assert np.linalg.norm(f64(got) - exact) <= tol * np.linalg.norm(exact)
    step = oracle.orthogonalise(f64(out["dW"]), 5, (3.4445, -4.7750, 2.0315))
    assert np.linalg.norm(f64(out["step"]) - step) <= (5.6e-3 + 2.0 ** -8 / 3 ** 0.5) * np.linalg.norm(step)


def test_two_graphs_with_workspaces_of_their_own_replay_at_once():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    M, K, N = 200, 256, 700
    bf = torch.bfloat16
    cases = []
    for i in range(2):
        x, W = (torch.randn((M, K), generator=g, device=DEV)).to(bf), (torch.randn((N, K), generator=g, device=DEV) / 16).to(bf)
        label = torch.randint(0, N, (M,), generator=g, device=DEV).int()
        loss, lse = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
        dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty(N, device=DEV)
        dloss = torch.ones(M, device=DEV)
        ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (
            som.som_cross_entropy_workspace_bytes(M, N, K), som.som_cross_entropy_backward_workspace_bytes(M, N, K),
            som.som_orthogonalise_workspace_bytes(N, K))]
        step = torch.empty_like(W)

        def run(x=x, W=W, label=label, loss=loss, lse=lse, dx=dx, dW=dW, db=db, dloss=dloss, ws=ws, step=step):
            som.som_cross_entropy(x, W.t(), label, loss=loss, lse=lse, ws=ws[0])
            som.som_cross_entropy_backward(dloss, x, W.t(), label, lse, dx=dx, dW=dW.t(), dbias=db, ws=ws[1])
            som.som_orthogonalise(dW, y=step, ws=ws[2])

        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (loss, lse, dx, dW, db, step)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        # (a graph does not keep its tensors: `run` does)
        cases.append((graph, (loss, lse, dx, dW, db, step), want, torch.cuda.Stream(), run))
    for _ in range(3):
        for _, got, _, _, _ in cases:
            for t in got:
                t.zero_()
        torch.cuda.synchronize()
        for graph, _, _, stream, _ in cases:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, got, want, _, _ in cases:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_threads_on_streams_of_their_own_get_their_own_results():
    import threading

    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    bf = torch.bfloat16
    sizes = [(200, 256, 700), (131, 384, 1000)]
    cases = []
    for M, K, N in sizes:
        x = torch.randn((M, K), generator=g, device=DEV).to(bf)
        W = (torch.randn((N, K), generator=g, device=DEV) / 16).to(bf)
        label = torch.randint(0, N, (M,), generator=g, device=DEV).int()
        dloss = torch.rand(M, generator=g, device=DEV)

        def run(stream, x=x, W=W, label=label, dloss=dloss):
            loss, lse = som.som_cross_entropy(x, W.t(), label, stream=stream)
            dx, dW, db = som.som_cross_entropy_backward(dloss, x, W.t(), label, lse, stream=stream)
            step = som.som_orthogonalise(dW.t(), stream=stream)
            q, s = som.som_quantise(x, stream=stream)
            w, ws = som.som_quantise(step, 128, stream=stream)
            return loss, lse, dx, dW, db, step, som.som_product_blocks(q, s, w.t(), ws, stream=stream)

        want = run(None)
        torch.cuda.synchronize()
        cases.append((run, want, torch.cuda.Stream()))
    got = [None, None]

    def work(i):
        run, _, stream = cases[i]
        got[i] = [run(stream) for _ in range(20)]

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for (_, want, _), results in zip(cases, got):
        assert results is not None
        for result in results:
            assert all(torch.equal(a, b) for a, b in zip(result, want))
