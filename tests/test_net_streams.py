"""The scratch that a call allocates for itself belongs to the stream that the call
runs on: a block of the current stream's may still be in use there, and nothing
orders another stream behind that."""
import pytest
import torch

from host_tensors import Library, Streams, gpu, on_host_device


@pytest.fixture
def evox(monkeypatch):
    import paper_2301_12457_amd as m
    L = Library()
    monkeypatch.setattr(m, "lib", lambda: L)
    m.calls = L.calls
    on_host_device(m, monkeypatch)
    return m


def calls(evox):
    x, w, dy, v = gpu(torch.zeros(6, 4)), gpu(torch.zeros(2, 3, 4)), gpu(torch.zeros(6, 3)), gpu(torch.zeros(6))
    p, lab, fit = gpu(torch.zeros(2, 4)), gpu(torch.zeros(6, dtype=torch.int32)), gpu(torch.zeros(2))
    return {"evox_linear_grad": lambda s: evox.evox_linear_grad(x, w, dy, dw=w.clone(), stream=s),
            "evox_layernorm_grad": lambda s: evox.evox_layernorm_grad(x, p, v, v, x, dx=x.clone(), stream=s),
            "evox_xent": lambda s: evox.evox_xent(x, lab, fit, stream=s)}


@pytest.mark.parametrize("name", ["evox_linear_grad", "evox_layernorm_grad", "evox_xent"])
def test_scratch_of_the_call_s_stream(evox, monkeypatch, name):
    streams = Streams(monkeypatch)
    side = streams.stream(2)
    calls(evox)[name](side)
    assert [s.cuda_stream for s in streams.allocated] == [2]
    (called, args), = [c for c in evox.calls if c[0] == name]
    assert args[-1] == 2 and streams.now.cuda_stream == 1


def test_scratch_of_the_sort_s_stream(evox, monkeypatch):
    streams = Streams(monkeypatch)
    evox.evox_nsga2_sort(gpu(torch.zeros(8, 3)), gpu(torch.zeros(8, dtype=torch.int32)),
                         gpu(torch.zeros(8, dtype=torch.float64)), stream=streams.stream(2))
    assert [s.cuda_stream for s in streams.allocated] == [2]
    (called, args), = [c for c in evox.calls if c[0] == "evox_nsga2_sort"]
    assert args[-2] >= 4096 and args[-1].value == 2


def test_a_state_waits_for_the_memory_it_takes(evox, monkeypatch):
    """Its buffers are the current stream's, its kernels may run on another: behind
    what is pending there."""
    streams = Streams(monkeypatch)
    params = evox.Params(algo=evox.PSO, fn_id=0, N=8, D=4, ldx=4)
    for stream, waited in ((streams.stream(2), [(2, 1)]), (None, []), (streams.now, [])):
        streams.waited.clear()
        evox.Swarm(params, stream=stream)
        assert streams.waited == waited
