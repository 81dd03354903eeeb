"""Which kernels the layers' tests reach (host arithmetic): a change of the rules
that choose them must not empty a test unseen."""
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


def test_every_shape_of_every_product(evox):
    """With sums of several K tiles, so that the tile two ahead is loaded in time."""
    import test_gpu_linear_tiles as t
    for dt in (evox.F32, evox.BF16, evox.F16):
        reached = [set(), set(), set()]
        for G, mean, n_in, n_out in t.CASES:
            kernels = evox.layer_kernels(dt, G, G * mean, n_in, n_out, ragged=True)
            for product, K in enumerate((n_in, n_out, mean)):
                if K > 200:
                    reached[product].add(kernels[product])
        shapes = {evox.KERNEL_TILES + i for i in range(4)}
        shares = {evox.KERNEL_TILES + evox.KERNEL_SHARES}
        assert shapes <= reached[0] and shapes | shares <= reached[1] and shapes | shares <= reached[2], (dt, reached)
        for i, kernels in t.EVEN.items():
            G, n, n_in, n_out = t.CASES[i]
            assert list(evox.layer_kernels(dt, G, G * n, n_in, n_out)) == kernels[dt != evox.F32]


def test_gradients_of_every_kind(evox):
    """The gradient's one-rounding test covers each way that a 16-bit one takes."""
    import test_gpu_linear_grad_bits as t
    reached = set()
    for counts, n_in, n_out in t.CASES:
        reached.update(enumerate(evox.layer_kernels(evox.BF16, len(counts), sum(counts), n_in, n_out, ragged=True)[1:]))
    for product in (0, 1):
        for kind in (evox.KERNEL_NARROW, evox.KERNEL_FEW_INPUTS, evox.KERNEL_SHORT, evox.KERNEL_TILES,
                     evox.KERNEL_TILES + evox.KERNEL_SHARES):
            assert (product, kind) in reached, (product, kind, reached)


def test_kernels_refuse(evox):
    L, out = evox.lib(), [ctypes.byref(ctypes.c_int32(0)) for _ in range(3)]
    good = evox.Layer(evox.F32, 0, 2, 6, 4, 3)
    assert L.evox_layer_kernels(ctypes.byref(good), *out) == evox.OK
    assert L.evox_layer_kernels(None, *out) == evox.EINVAL
    assert L.evox_layer_kernels(ctypes.byref(good), out[0], None, out[2]) == evox.EINVAL
    with pytest.raises(evox.EvoxError):
        evox.layer_kernels(evox.F32, 4, 6, 4, 3)
    with pytest.raises(evox.EvoxError):
        evox.layer_kernels(3, 2, 6, 4, 3)


def test_pairs_of_both_kinds(evox):
    import test_gpu_linear_grad_bits as t
    reached = {evox.layer_kernels(dt, len(counts), sum(counts), n_in, n_out, len(set(counts)) > 1, evox.ACT_GELU)[1]
               for counts, n_in, n_out in t.PAIRS for dt in (evox.BF16, evox.F16)}
    assert {evox.KERNEL_TILES + 4, evox.KERNEL_TILES + 4 + evox.KERNEL_SHARES} <= reached, reached
