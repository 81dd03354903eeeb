"""Tensors of the host that say they are on the GPU, and a library that only notes
its calls: what the binding does with a call, where there is no GPU."""
import types

import torch


class OnGpu(torch.Tensor):
    """A host tensor whose get_device() is a GPU's."""
    index = 0

    def get_device(self):
        return self.index

    def record_stream(self, stream):
        pass


def gpu(t, index=0):
    t = t.as_subclass(OnGpu)
    t.index = index
    return t


class Library:
    """Every function notes (name, arguments); sizes are 4096, everything else 0."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 4096 if name.endswith("_bytes") else 0
        return call


class Streams:
    """torch.cuda's current stream and torch.empty, noted: which stream was current
    at each allocation."""

    def __init__(self, monkeypatch, device=0):
        self.now, self.allocated, self.waited = self.stream(1, device), [], []
        real = torch.empty

        def empty(*args, **kw):
            self.allocated.append(self.now)
            kw.pop("device", None)
            return gpu(real(*args, **kw), device)

        monkeypatch.setattr(torch, "empty", empty)
        monkeypatch.setattr(torch.cuda, "stream", self.use)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.now)

    def stream(self, handle, device=0):
        return types.SimpleNamespace(cuda_stream=handle, device_index=device, device=torch.device("cuda", device),
                                     wait_stream=lambda other: self.waited.append((handle, other.cuda_stream)))

    def use(self, stream):
        outer = self

        class Context:
            def __enter__(self):
                self.before, outer.now = outer.now, stream if stream is not None else outer.now

            def __exit__(self, *args):
                outer.now = self.before
        return Context()


def on_host_device(evox, monkeypatch, current=0):
    """The binding with this current device, whose current stream is 7."""
    evox._look_at_torch()
    monkeypatch.setattr(evox, "_DTYPES", dict(evox._DTYPES, stream=lambda device: 7, device=lambda: current))
