"""The binding of the networks' operators, on the host: tensors that say they are on
the GPU and a library that notes its calls stand in for both."""
import pytest
import torch

from host_tensors import Library, Streams, gpu, on_host_device


@pytest.fixture
def evox(monkeypatch):
    import paper_2301_12457_amd as m
    L = Library()
    monkeypatch.setattr(m, "lib", lambda: L)
    m.calls = L.calls
    return m


def test_first_call_from_two_threads(evox, monkeypatch):
    """A call that comes while another one's first look at torch is under way finds
    either nothing there or all of it."""
    x, v = gpu(torch.zeros(6, 4)), gpu(torch.zeros(6))
    inside = []

    class Table(dict):
        def probe(self):
            if not inside:
                inside.append(1)
                assert evox._dtype(x) == evox.F32 and evox._vector("v", v, "float32", 6, x) == v.data_ptr()
                assert evox._DTYPES["stream"]
                inside.clear()

        def update(self, *a, **k):
            super().update(*a, **k)
            self.probe()

        def __setitem__(self, k, v):
            super().__setitem__(k, v)
            self.probe()

    monkeypatch.setattr(evox, "_DTYPES", Table())
    assert evox._dtype(x) == evox.F32
    assert evox._vector("v", v, "float32", 6, x) == v.data_ptr()


@pytest.mark.parametrize("tensors,current,stream,fits", [(0, 0, None, True), (0, 0, 0, True), (1, 0, None, False),
                                                         (0, 1, None, False), (1, 1, 1, True), (1, 1, 0, False),
                                                         (1, 0, 1, False), (0, 0, 1, False)])
def test_another_device_than_the_stream_s(evox, monkeypatch, tensors, current, stream, fits):
    """A kernel runs on its stream's device, and a stream's handle alone (0 for every
    default one) leaves that to the current device."""
    on_host_device(evox, monkeypatch, current)
    new = lambda *shape, **kw: gpu(torch.zeros(*shape, **kw), tensors)
    x, w, y, v, p = new(6, 4), new(2, 3, 4), new(6, 3), new(6), new(2, 4)
    lab, fit, scratch = new(6, dtype=torch.int32), new(2), new(4096)
    s = None if stream is None else Streams(monkeypatch).stream(5, stream)
    for call in (lambda: evox.evox_linear(x, w, y, stream=s), lambda: evox.evox_linear_grad(x, w, y, dx=new(6, 4), scratch=scratch, stream=s),
                 lambda: evox.evox_layernorm(x, p, p, new(6, 4), stream=s),
                 lambda: evox.evox_layernorm_grad(x, p, v, v, x, dx=new(6, 4), scratch=scratch, stream=s),
                 lambda: evox.evox_xent(x, lab, fit, scratch=scratch, stream=s)):
        evox.calls.clear()
        if fits:
            call()
            assert evox.calls[-1][1][-1] == (7 if stream is None else 5)
        else:
            with pytest.raises(evox.EvoxError, match="device"):
                call()
            assert all(name.endswith("_bytes") for name, _ in evox.calls)
