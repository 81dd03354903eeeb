"""Scratch sizes: what the query answers covers a call with and without offsets
(host arithmetic only).  And tensors that are not on the GPU are refused."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def evox():
    import paper_2301_12457_amd as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2301_12457_amd import build
        build.build()
    return m


P = 0x1000  # never dereferenced
SIZES = [(1, 1), (1, 64), (1, 100_000), (7, 7 * 64), (515, 515 * 140), (600, 600 * 3000), (512, 512 * 64), (2048, 2048 * 70),
         (5000, 5000), (448, 448 * 65), (300, 300 * 64), (100, 100 * 330)]


@pytest.mark.parametrize("G,M", SIZES)
def test_scratch_without_offsets(evox, G, M):
    L = evox.lib()
    for dt in (evox.F32, evox.BF16):
        for i, o in ((5, 33), (8, 1), (32, 65), (20, 1109), (64, 64), (33, 900), (700, 2), (1000, 1000)):
            a = [L.evox_linear_grad_scratch_bytes(ctypes.byref(evox.Layer(
                dt, 0, G, M, i, o, off, 0, i, i, i * o, o, o, o, o, i, i, i * o, o))) for off in (None, P)]
            assert a[0] == a[1] > 0, (G, M, i, o, a)
        for D in (3, 100, 5000):
            a = [L.evox_layernorm_grad_scratch_bytes(ctypes.byref(evox.Norm(dt, G, M, D, off, D, D, D, D, D, 1e-5)))
                 for off in (None, P)]
            assert a[0] == a[1] > 0, (G, M, D, a)


def test_tensors_of_the_host_are_refused(evox):
    import torch
    x, w, y, v = torch.zeros(6, 4), torch.zeros(2, 3, 4), torch.zeros(6, 3), torch.zeros(6)
    for call in (lambda: evox.evox_linear(x, w, y), lambda: evox.evox_linear_grad(x, w, y, dx=x),
                 lambda: evox.evox_linear_grad_scratch(x, w, y),
                 lambda: evox.evox_layernorm(x, x[:2], x[:2], x), lambda: evox.evox_layernorm_grad(x, x[:2], v, v, x, dx=x),
                 lambda: evox.evox_xent(x, torch.zeros(6, dtype=torch.int32), v[:2])):
        with pytest.raises(evox.EvoxError) as e:
            call()
        assert e.value.args
