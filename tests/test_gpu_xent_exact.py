"""The cross-entropy's fitness is the same bits with and without the gradient, NaN
(networks without a counted row) in the same places."""
import pytest
import torch

import net_ref as nr
from test_gpu_norm import XSHAPES, check_xent, xent_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(XSHAPES)))
def test_fitness_alone(evox_gpu, dtype, i):
    counts, C = XSHAPES[i]
    print(f"xent alone {dtype} {counts[:6]} {C}", flush=True)
    s = xent_inputs(dtype, counts + [0, 1], C, pad=i % 3, seed=i, ignore=0.1)
    s["labels"][-1] = -1
    fit, _ = check_xent(evox_gpu, s, pad=i % 3)
    alone, _ = check_xent(evox_gpu, s, grad=False)
    assert torch.isnan(fit[-2:]).all()
    assert torch.equal(torch.isnan(fit), torch.isnan(alone))
    assert torch.equal(fit[~torch.isnan(fit)], alone[~torch.isnan(fit)])
