"""The binding of the networks' operators, on the host: tensors that say they are on
the GPU and a library that notes its calls stand in for both."""
import pytest
import torch

from host_tensors import Library, gpu


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
