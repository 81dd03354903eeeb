"""Calls on another stream than the current one, with the scratch that they allocate
themselves: the same bits, and work that is pending on the current stream keeps
the memory it reads."""
import pytest
import torch

import net_ref as nr
from test_gpu_linear import layer
from test_gpu_norm import norm_inputs, xent_inputs

pytestmark = pytest.mark.gpu


def calls(ev):
    s = layer(torch.bfloat16, [100, 0, 57, 300], 160, 136, seed=5)
    n = norm_inputs(torch.float32, [70, 0, 300], 260, seed=4)
    x = xent_inputs(torch.float32, [300, 17, 64], 500, seed=13)
    like = lambda t, *shape: torch.empty(shape or t.shape, dtype=t.dtype, device="cuda")
    stat = torch.rand(n["M"], generator=torch.Generator().manual_seed(1)).cuda()

    def linear_grad(out, stream):
        ev.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=out[0], dw=out[1], db=out[2], off=s["off"],
                            act=ev.ACT_GELU, stream=stream)

    def layernorm_grad(out, stream):
        ev.evox_layernorm_grad(n["x"], n["gamma"], stat, stat, n["dy"], *out, off=n["off"], stream=stream)

    def xent(out, stream):
        ev.evox_xent(x["z"], x["labels"], out[0], dz=out[1], off=x["off"], stream=stream)

    # the calls and their outputs
    return {"linear_grad": (linear_grad, [like(s["x"]), like(s["w"], *s["w"].shape), like(s["b"], *s["b"].shape)]),
            "layernorm_grad": (layernorm_grad, [like(n["x"], n["M"], n["D"]), *(like(n["x"], n["G"], n["D"]) for _ in "gb")]),
            "xent": (xent, [torch.empty(x["G"], device="cuda"), like(x["z"], x["M"], x["C"])])}


@pytest.mark.parametrize("name", ["linear_grad", "layernorm_grad", "xent"])
def test_side_stream_with_its_own_scratch(evox_gpu, name):
    call, out = calls(evox_gpu)[name]
    call(out, None)
    want = [t.clone() for t in out]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.randn(2048, 2048, device="cuda")
    for n in (1 << 12, 1 << 14, 1 << 16, 1 << 18, 1 << 20, 1 << 22):  # freed blocks of every size the scratch could take
        held = [torch.full((n,), 3, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        for _ in range(8):
            busy = (busy @ busy).clamp(-1, 1)
        copies = [t.clone() for t in held]  # behind the products
        del held
        call(out, side)
        torch.cuda.synchronize()
        assert all((t == 3).all() for t in copies)
        assert all(torch.equal(p, q) for p, q in zip(out, want))
        for t in out:
            t.fill_(float("nan"))


def test_sort_on_a_side_stream(evox_gpu):
    F = torch.rand(700, 3, generator=torch.Generator().manual_seed(2)).cuda()
    new = lambda: (torch.empty(700, dtype=torch.int32, device="cuda"), torch.empty(700, dtype=torch.float64, device="cuda"))
    want, got = new(), new()
    evox_gpu.evox_nsga2_sort(F, *want)
    torch.cuda.synchronize()
    evox_gpu.evox_nsga2_sort(F, *got, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_a_state_on_a_side_stream(evox_gpu):
    """A state on another stream, started behind pending readers of freed memory."""
    params = evox_gpu.make_params(evox_gpu.PSO, evox_gpu.SPHERE, 512, 64, -5.0, 5.0, seed=3)
    want = evox_gpu.Swarm(params)
    want.step(3)
    torch.cuda.synchronize()
    busy = torch.randn(2048, 2048, device="cuda")
    held = [torch.full((512 * 64,), 3.0, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    for _ in range(8):
        busy = (busy @ busy).clamp(-1, 1)
    copies = [t.clone() for t in held]
    del held
    got = evox_gpu.Swarm(params, stream=torch.cuda.Stream())
    got.step(3)
    torch.cuda.synchronize()
    assert all((t == 3).all() for t in copies)
    assert torch.equal(got.view("x"), want.view("x")) and torch.equal(got.gbest, want.gbest)
