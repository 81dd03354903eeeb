"""The tests' buffers of NaN are written before a call on another stream can write its results."""
import pytest
import torch

from test_gpu_linear import filled

pytestmark = pytest.mark.gpu


def test_filled_is_done(evox_gpu):
    busy = torch.randn(4096, 4096, device="cuda")
    for _ in range(20):
        busy = (busy @ busy).clamp(-1, 1)
    y = filled(300, 200, torch.bfloat16, 3)  # behind the products
    assert torch.cuda.current_stream().query()
    assert y.shape == (300, 200) and y.isnan().all()
