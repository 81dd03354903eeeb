"""Networks of many row tiles (their sums are joined by many threads), networks that
are one tile each, long sums shared by waves, and rows over every number of
lanes, against 64 bits on the GPU.  Bounds as in the layers' and norms' tests."""
import pytest

import net_ref as nr
from test_gpu_linear import check_grad, layer
from test_gpu_linear_large import check_all
from test_gpu_norm import check_norm, check_norm_grad, check_xent, norm_inputs, xent_inputs

pytestmark = pytest.mark.gpu

# rows, n_in, n_out, activation, same rows for each network
LAYERS = [([70_000], 9, 130, "tanh", False), ([30_000, 0, 17, 1500], 20, 24, "gelu", False), ([40_000], 3, 1, "none", False),
          ([128] * 600, 16, 16, "silu", True), ([70] * 520, 40, 33, "tanh", True), ([300, 0, 41] * 4, 64, 64, "gelu", False),
          ([300, 0, 41] * 4, 48, 64, "relu", False), ([1] * 5, 4100, 40, "none", False), ([7, 0, 20], 2100, 33, "silu", False),
          ([30, 32] * 3, 600, 100, "none", False), ([26, 40], 70, 120, "tanh", False), ([3000], 1100, 18, "gelu", False),
          ([600] * 512, 8, 1, "tanh", True), ([150] * 520, 20, 24, "silu", True), ([140] * 515, 5, 33, "gelu", False),
          ([300, 0, 41, 64, 1] * 3, 18, 200, "gelu", False), ([70] * 40, 1, 77, "none", False), ([5000], 16, 700, "silu", False), ([33_000], 20, 1109, "gelu", False),
          ([128] * 4, 32, 65, "tanh", True), ([64] * 5, 7, 130, "relu", True), ([2] * 30, 9, 300, "silu", False)]


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(LAYERS)))
def test_layers(evox_gpu, dtype, i):
    counts, n_in, n_out, act, even = LAYERS[i]
    print(f"layers {dtype} {counts[:4]} x{len(counts)} {n_in}x{n_out} {act}", flush=True)
    check_all(evox_gpu, layer(dtype, counts, n_in, n_out, lead=i % 3, even=even, resid=True, seed=50 + i), act, f"case {i}")


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("G,n,n_in,n_out", [(5, 70, 20, 100), (3, 64, 5, 67)])
def test_shared_rows(evox_gpu, dtype, G, n, n_in, n_out):
    print(f"shared {dtype} {G}x{n} {n_in}x{n_out}", flush=True)
    check_grad(evox_gpu, layer(dtype, [n] * G, n_in, n_out, lead=1, pad=1, shared=True, seed=G), "gelu", pad=1)


NORMS = [([20_000], 40), ([9000, 0, 1, 700], 12), ([50, 3], 250), ([90], 136), ([30, 2], 8192), ([300, 0, 9], 4100), ([2500], 600)]


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(NORMS)))
def test_norms(evox_gpu, dtype, i):
    counts, D = NORMS[i]
    print(f"norms {dtype} {counts} x {D}", flush=True)
    s = norm_inputs(dtype, counts, D, pad=i % 3, lead=i % 2, seed=60 + i)
    check_norm(evox_gpu, s)
    check_norm_grad(evox_gpu, s)


LOSSES = [([20_000, 0, 3], 10), ([3000], 600), ([400, 9], 136), ([31], 9000), ([5] * 30, 250)]


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(LOSSES)))
def test_losses(evox_gpu, dtype, i):
    counts, C = LOSSES[i]
    print(f"losses {dtype} {counts[:3]} x {C}", flush=True)
    check_xent(evox_gpu, xent_inputs(dtype, counts, C, pad=i % 3, seed=70 + i))
