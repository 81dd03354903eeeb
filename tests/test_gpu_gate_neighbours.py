"""What a row of the gate's results is does not depend on the other rows of its batch, to the
last bit: rows of NaN, infinities and large logits beside it."""
import math

import pytest
import torch

from net_ref import DTYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("over", [0, 1])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", [(64, 2, 2), (500, 9, 3), (4000, 32, 8), (3000, 64, 2), (2000, 100, 5), (1000, 256, 8), (9000, 256, 4), (300, 1000, 32),
                                   (5000, 2048, 3), (40, 4099, 5)])
def test_rows_by_themselves(evox_gpu, T, G, k, dtype, over):
    rng = torch.Generator().manual_seed(T + G)
    z = (torch.randn(T, G, generator=rng) * 5).to(dtype).cuda()
    dw = torch.randn(T, k, generator=rng).cuda()

    def run(z):
        ids, w, dz = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda"), torch.empty_like(z)
        evox_gpu.evox_gate(z, ids, w, over=over)
        evox_gpu.evox_gate_grad(z, ids, w, dw, dz, over=over)
        return ids, w, dz

    want = run(z)
    odd = torch.rand(T, generator=rng) < 0.15
    large = 60_000.0 if dtype is torch.float16 else 1e30
    beside = z.clone()
    for i, t in enumerate(odd.nonzero().flatten().tolist()):
        beside[t, i % G] = (math.nan, math.inf, large, -large)[i % 4]
        if i % 8 == 7:
            beside[t] = -math.inf
    rest = (~odd).cuda()
    for a, b in zip(want, run(beside)):
        assert torch.equal(a[rest], b[rest])
