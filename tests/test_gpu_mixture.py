"""The mixture's operators together, as examples/mixture_of_networks.py uses them: its
gradients against 64-bit autograd, eagerly, on another stream and captured."""
import importlib.util
import os

import pytest
import torch

from net_ref import DTYPES, U

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example(evox_gpu):
    spec = importlib.util.spec_from_file_location("mixture_of_networks", os.path.join(ROOT, "examples", "mixture_of_networks.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(net, x, dy, ids):
    """y and the parameters' gradients in 64 bits, with the choices that were made."""
    p = {n: v.double().cpu().requires_grad_() for n, v in net.params.items()}
    x = x.double().cpu()
    h = torch.tanh(x @ p["w0"][0].t() + p["b0"][0])
    logits = h @ p["wg"][0].t() + p["bg"][0]
    ids = ids.cpu().long()
    w = torch.softmax(logits, 1).gather(1, ids) if net.over else torch.softmax(logits.gather(1, ids), 1)
    act = torch.nn.functional.gelu(torch.einsum("ti,tjoi->tjo", h, p["w1"][ids]) + p["b1"][ids])
    ys = torch.einsum("tjh,tjch->tjc", act, p["w2"][ids]) + p["b2"][ids]
    y = (w[:, :, None] * ys).sum(1)
    y.backward(dy.double().cpu())
    return y.detach(), logits.detach(), {n: v.grad for n, v in p.items()}


def near(got, want, dtype, what):
    """A handful of layers, each rounded to the type, over sums of hundreds of rows with
    errors of either sign: 40 roundings of the largest of a tensor's numbers."""
    got = got.double().cpu()
    off = (got - want).abs().max() / want.abs().max().clamp_min(1e-6)
    assert off <= 40 * U[dtype], (what, float(off))


@pytest.mark.parametrize("over", [0, 1])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", [(1, 8, 2), (333, 8, 2), (500, 5, 5), (64, 40, 1)])
def test_gradients(example, T, G, k, dtype, over):
    net = example.Mixture(T, G=G, k=k, dtype=dtype, over=over, seed=T)
    rng = torch.Generator(device="cuda").manual_seed(1)
    x, dy = torch.randn(T, 10, generator=rng, device="cuda").to(dtype), torch.randn(T, 6, generator=rng, device="cuda").to(dtype)
    net.forward(x)
    net.backward(x, dy)
    y, logits, grads = reference(net, x, dy, net.ids)
    # the choices are the largest logits, but for ones that roundings may have swapped
    chosen = logits.gather(1, net.ids.cpu().long())
    kth = torch.topk(logits, k, 1).values[:, -1:]
    assert (chosen >= kth - 40 * U[dtype] * logits.abs().max()).all()
    near(net.y, y, dtype, "y")
    for name, g in grads.items():
        near(net.grads[name], g, dtype, name)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_and_on_another_stream(evox_gpu, example, dtype):
    """Steps by a graph, and by a stream of their own, are the eager steps bit for bit."""
    T, runs = 400, []
    for how in range(3):
        net = example.Mixture(T, dtype=dtype, seed=3)
        opt = evox_gpu.AdamW(net.X, net.dX, lr=1e-2, bits=8, master=dtype is torch.bfloat16)
        x, labels = (t.clone() for t in example.data(T, "cuda", 0))
        x = x.to(dtype)
        side = torch.cuda.Stream()
        losses = [net.train(x, labels, opt).clone()]
        graph = torch.cuda.CUDAGraph()
        if how == 1:
            with torch.cuda.graph(graph):
                net.train(x, labels, opt)
        for i in range(1, 5):
            a, b = example.data(T, "cuda", i)
            x.copy_(a)
            labels.copy_(b)
            if how == 0:
                net.train(x, labels, opt)
            elif how == 1:
                graph.replay()
            else:
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    net.train(x, labels, opt)
                torch.cuda.current_stream().wait_stream(side)
            losses.append(net.loss.clone())
            float(torch.cat(losses).sum())  # the program's own work and waits between replays
        runs.append((torch.cat(losses), [p.clone() for p in net.X], opt.state["t"].item()))
    for losses, X, t in runs[1:]:
        assert torch.equal(losses, runs[0][0]) and t == runs[0][2] == 5
        assert all(torch.equal(a, b) for a, b in zip(X, runs[0][1]))


def test_example_runs(example):
    for bits, dtype in ((32, torch.float32), (8, torch.bfloat16)):
        losses = example.run(steps=4, T=256, bits=bits, dtype=dtype)
        assert len(losses) == 4 and all(l == l and abs(l) < 100 for l in losses)


def test_calls_on_a_given_stream(evox_gpu):
    """Each call's stream argument: results come after what that stream has before."""
    evox = evox_gpu
    T, G, k, D = 5000, 300, 4, 257
    rng = torch.Generator(device="cuda").manual_seed(0)
    z, x = torch.randn(T, G, generator=rng, device="cuda"), torch.randn(T, D, generator=rng, device="cuda")
    new = lambda *s, d=torch.float32: torch.zeros(*s, dtype=d, device="cuda")

    def run(stream):
        zz, xx = new(T, G), new(T, D)
        ids, w, off, pos = new(T, k, d=torch.int32), new(T, k), new(G + 1, d=torch.int32), new(T, k, d=torch.int32)
        xs, y, dxs, dw, dz = new(T * k, D), new(T, D), new(T * k, D), new(T, k), new(T, G)
        p, g = x.clone(), x.clone()
        opt = evox.AdamW([p], [g])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            zz.copy_(z)
            xx.copy_(x)
        evox.evox_gate(zz, ids, w, over=1, stream=stream)
        evox.evox_route(ids, off, pos, stream=stream)
        evox.evox_dispatch(xx, pos, xs, w=w, stream=stream)
        evox.evox_combine(xs, pos, y, w=w, r=xx, stream=stream)
        evox.evox_combine_grad(xs, pos, y, w=w, dxs=dxs, dw=dw, stream=stream)
        evox.evox_gate_grad(zz, ids, w, dw, dz, over=1, stream=stream)
        opt.step(stream=stream)
        torch.cuda.synchronize()
        return ids, w, off, pos, xs, y, dxs, dw, dz, p

    for a, b in zip(run(None), run(torch.cuda.Stream())):
        assert torch.equal(a, b)
