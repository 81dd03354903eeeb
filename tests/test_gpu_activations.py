"""Activations and their slopes one element at a time (layers 1 x 1 of weight 1):
infinities and NaN alike in all types, and the small ends to the type's own
rounding.

Bounds, relative: the argument's square is rounded once where an exponential
takes it, 2 u z^2 of it, u = 2^-24; a published or fitted polynomial, a
reciprocal and the products 2^-15 in 16 bits, far below the type's roundoff, and
16 u in fp32."""
import math

import pytest
import torch

import net_ref as nr

pytestmark = pytest.mark.gpu
INF = float("inf")
VALUES = {"none": (INF, -INF), "relu": (INF, 0.0), "tanh": (1.0, -1.0), "gelu": (INF, 0.0), "silu": (INF, 0.0)}
SLOPES = {"none": (1.0, 1.0), "relu": (1.0, 0.0), "tanh": (0.0, 0.0), "gelu": (1.0, 0.0), "silu": (1.0, 0.0)}


def value_and_slope(ev, z, act):
    one = torch.ones(1, 1, 1, dtype=z.dtype, device="cuda")
    y, dx = torch.empty_like(z), torch.empty_like(z)
    ev.evox_linear(z, one, y, act=nr.ACTS.index(act))
    ev.evox_linear_grad(z, one, torch.ones_like(z), z=z, dx=dx, act=nr.ACTS.index(act))
    return y, dx


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("act", nr.ACTS)
def test_infinities_and_nan(evox_gpu, dtype, act):
    z = torch.tensor([INF, -INF, float("nan"), 1.0], device="cuda").to(dtype)[:, None]
    y, dx = value_and_slope(evox_gpu, z, act)
    assert y[:2, 0].tolist() == list(VALUES[act]) and dx[:2, 0].tolist() == list(SLOPES[act])
    assert math.isnan(float(y[2])) and (act == "none" or math.isnan(float(dx[2])))
    assert math.isfinite(float(y[3])) and math.isfinite(float(dx[3]))


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_infinities_through_tiles(evox_gpu, dtype, act):
    """The same behind the layers' large products (their sums are -inf, inf and NaN)."""
    G, n, n_in, n_out = 6, 300, 130, 520
    x, w = torch.zeros(G * n, n_in, device="cuda", dtype=dtype), torch.ones(G, n_out, n_in, device="cuda", dtype=dtype)
    x[1, 3], x[2, 4], x[5, 5], x[n + 7, 8] = -INF, INF, float("nan"), -INF
    y = torch.empty(G * n, n_out, device="cuda", dtype=dtype)
    evox_gpu.evox_linear(x, w, y, act=nr.ACTS.index(act))
    want = torch.zeros(G * n, n_out, device="cuda", dtype=dtype)
    want[2], want[5] = INF, float("nan")
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y[~torch.isnan(want)], want[~torch.isnan(want)])


def check_small_ends(evox_gpu, dtype, act):
    """Values and slopes from -12 to 12 relative to themselves (slopes of GELU and
    SiLU, which cross zero, to the sum of their terms)."""
    z = torch.linspace(-12, 12, 20_001, device="cuda").to(dtype)[:, None]
    y, dx = value_and_slope(evox_gpu, z, act)
    zz = z.double()
    want, slope = nr.act64(zz, act), nr.slope64(zz, act)
    rel = (16 * nr.U32 if dtype == torch.float32 else 2.0 ** -15) + 4 * nr.U32 * zz * zz
    terms = slope
    if act == "gelu":
        terms = 0.5 * torch.erfc(-zz / math.sqrt(2)) + zz.abs() * torch.exp(-zz * zz / 2) / math.sqrt(2 * math.pi)
    elif act == "silu":
        s = torch.sigmoid(zz)
        terms = s * (1 + zz.abs() * torch.sigmoid(-zz))
    for got, exact, scale in ((y, want, want.abs()), (dx, slope, terms)):
        limit = rel * scale + (exact.abs() + rel * scale) * nr.U[dtype] * 1.0001 + nr.TINY[dtype]
        bad = ~((got.double() - exact).abs() <= limit)
        assert not bad.any(), (f"{act} {dtype}: {int(bad.sum())} off, e.g. at {z[bad][:3].tolist()}: {got[bad][:3].tolist()} for "
                               f"{exact[bad][:3].tolist()} +- {limit[bad][:3].tolist()}")


@pytest.mark.parametrize("act", ["gelu", "silu", "tanh"])
def test_small_ends_of_fp32(evox_gpu, act):
    check_small_ends(evox_gpu, torch.float32, act)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["gelu", "silu", "tanh"])
def test_small_ends_of_16_bits(evox_gpu, dtype, act):
    check_small_ends(evox_gpu, dtype, act)


def test_tanh_slope_of_fp32(evox_gpu):
    """No further from 64 bits (root of the mean square) than 1 - tanh^2 in fp32,
    where that does not cancel."""
    z = torch.linspace(-1, 1, 100_001, device="cuda")[:, None]
    exact = nr.slope64(z.double(), "tanh")
    rms = lambda t: float((t.double() - exact).square().mean().sqrt())
    plain = rms(1 - torch.tanh(z).square())
    own = rms(value_and_slope(evox_gpu, z, "tanh")[1])
    print(f"tanh slope rms {own:.3g}, plain {plain:.3g}", flush=True)
    assert own <= plain
