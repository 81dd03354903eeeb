"""An optimizer's states on other streams than the one that they were made on: their memory is
not given to others before the stream's work on them is done."""
import types

import pytest
import torch

from host_tensors import Library, OnGpu, Streams, gpu, on_host_device


@pytest.fixture
def here(monkeypatch):
    import paper_2301_12457_amd as m
    L, real = Library(), torch.zeros
    streams = Streams(monkeypatch)
    monkeypatch.setattr(m, "lib", lambda: L)
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: gpu(real(*a, **{x: y for x, y in k.items() if x != "device"})))
    on_host_device(m, monkeypatch)
    m._DTYPES["stream"] = lambda device: streams.now.cuda_stream
    m.streams, m.recorded = streams, []
    monkeypatch.setattr(OnGpu, "record_stream", lambda self, s: m.recorded.append((self.data_ptr(), s.cuda_stream)))
    monkeypatch.setattr(torch.cuda, "Stream", types.SimpleNamespace)
    return m


def optimizer(m, bits=8):
    return m.AdamW([torch.zeros(6, 300)], [torch.zeros(6, 300)], bits=bits)


def recorded(m, opt, stream):
    """Whether all that a step reads and writes of the optimizer's own is recorded on a stream."""
    return {(t.data_ptr(), stream) for t in (opt._clock, opt._table, *opt.state.values())} <= set(m.recorded)


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_on_the_current_stream(here, bits):
    opt = optimizer(here, bits)
    opt.step()
    assert not here.recorded  # on its own stream
    with torch.cuda.stream(here.streams.stream(2)):
        opt.step()
    assert recorded(here, opt, 2)
    n = len(here.recorded)
    with torch.cuda.stream(here.streams.stream(2)):
        opt.step()
    opt.step()
    assert len(here.recorded) == n  # (once for a stream)
    with torch.cuda.stream(here.streams.stream(3)):
        opt.step()
    assert recorded(here, opt, 3)


def test_steps_on_a_given_stream(here):
    opt = optimizer(here)
    opt.step(stream=here.streams.stream(2))
    assert recorded(here, opt, 2)
    # given one of another kind, a handle with it: the caller sees to that
    opt.step(stream=type("Handle", (), {"cuda_stream": 9})())
    assert 9 not in [s for _, s in here.recorded]
    with torch.cuda.stream(here.streams.stream(9)):
        opt.step()
    assert recorded(here, opt, 9)
    here.recorded.clear()
    # the stream that the states are of, given to a program whose current one is another
    own = here.streams.now
    with torch.cuda.stream(here.streams.stream(4)):
        opt.step(stream=own)
    assert not here.recorded


def test_load_on_the_current_stream(here):
    opt = optimizer(here)
    state = {name: t.clone() for name, t in opt.state.items()}
    opt.load(state)
    assert not here.recorded
    with torch.cuda.stream(here.streams.stream(5)):
        opt.load(state)
    assert recorded(here, opt, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("how", ["current", "given", "load"])
def test_dropped_behind_a_step(evox_gpu, how, bits):
    """Blocks of the states' sizes that are allocated when the optimizer is gone are not those that
    the pending step writes."""
    n = 1 << 20
    p, g = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    busy = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    opt = evox_gpu.AdamW([p], [g], bits=bits)
    for _ in range(2):
        opt.step()
    saved = {name: t.clone() for name, t in opt.state.items()}
    sizes = [(t.shape, t.dtype) for t in opt.state.values()] + [(opt._clock.shape, opt._clock.dtype), (opt._table.shape, opt._table.dtype)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            busy = (busy @ busy).clamp(-1, 1)  # the step waits behind these
        if how == "current":
            opt.step()
        elif how == "load":
            opt.load(saved)
    if how == "given":
        opt.step(stream=side)
    del opt
    others = [torch.full(shape, 3, dtype=torch.uint8, device="cuda") if d is torch.float8_e4m3fn else torch.full(shape, 3, dtype=d, device="cuda")
              for shape, d in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert all((t == 3).all() for t in others)
