"""Which elements share a scale of 8-bit moments is the parameter's shape's to say: those of a
row of its first dimension, however it and its gradient lie in memory.  (A dense parameter of up to
a group's 256 elements, in rows of fewer than the 8 of a lane, with a dense gradient, has one scale.)"""
import math

import pytest
import torch

from host_tensors import Library, gpu, on_host_device
from mix_ref import adamw64
from net_ref import DTYPES, TINY, U, U32

BLOCK = 256
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.05)
# of these the first two have as many scales by rows as through all elements
SHAPES = [(2, 250), (40, 250), (7, 1824), (6, 300), (5, 3, 100), (300, 33), (9, 512), (3, 1027), (130, 7), (17, 16), (8, 32), (2, 128), (3, 8), (2, 2, 4)]


def memory(lead, pad, shape, **kw):
    """Zeros of this shape; with a lead or pad, a view of the rows of a wider matrix."""
    n = math.prod(shape[1:])
    return torch.zeros(shape[0], lead + n + pad, **kw)[:, lead:lead + n].unflatten(1, shape[1:])


@pytest.fixture
def here(monkeypatch):
    import paper_2301_12457_amd as m
    L, real = Library(), torch.zeros
    monkeypatch.setattr(m, "lib", lambda: L)
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: gpu(real(*a, **{x: y for x, y in k.items() if x != "device"})))
    on_host_device(m, monkeypatch)
    m.calls = L.calls
    return m


@pytest.mark.parametrize("shape", SHAPES)
def test_scales_by_rows_whatever_the_strides(here, shape):
    G, n = shape[0], math.prod(shape[1:])
    for p, g in ((0, 0), (0, 3), (3, 0), (5, 2)):
        opt = here.AdamW([memory(p, p, shape)], [memory(g, 0, shape)], bits=8)
        assert opt.state["m_scale"].shape == opt.state["v_scale"].shape == (G * -(-n // BLOCK),)
        t = [c for c in here.calls if c[0] == "evox_adamw_plan"][-1][1][2][0]
        # (a row in whole groups may go on into the next)
        assert (t.rows, t.n) == (G, n) or (t.rows, t.n) == (1, G * n) and n % BLOCK == 0


def test_moments_of_32_bits_and_single_rows_are_one_row(here):
    for shape, bits in (((6, 300), 32), ((5, 3, 100), 32), ((1, 3000), 8), ((3000,), 8), ((9, 512), 8), ((0, 300), 8), ((4, 0), 8), ((3, 4), 8)):
        here.AdamW([torch.zeros(*shape)], [torch.zeros(*shape)], bits=bits)
        t = [c for c in here.calls if c[0] == "evox_adamw_plan"][-1][1][2][0]
        assert (t.rows, t.n) == (1, math.prod(shape))


# ---------------------------------------------------------------------------
# On the GPU
# ---------------------------------------------------------------------------
def held(opt, name, shape):
    """The numbers that a moment's bytes and scales stand for, by the parameter's shape."""
    G, n = shape[0], math.prod(shape[1:])
    q, s = opt.state[name].double().cpu().view(G, n), opt.state[name + "_scale"].double().cpu().view(G, -(-n // BLOCK))
    s = s.repeat_interleave(BLOCK, 1)[:, :n]
    return (q * s).view(shape), s.reshape(shape)


def steps(evox, p0, g0, where, dtype, count=3, state=None):
    """Parameters and optimizer after some steps, p and g with these leads and pads."""
    p, g = (memory(*at, tuple(p0.shape), dtype=dtype, device="cuda") for at in where)
    p.copy_(p0)
    opt = evox.AdamW([p], [g], bits=8, **HYPER)
    if state is not None:
        opt.load(state)
    for i in range(count):
        g.copy_(g0 * (1, -0.5, 0.25)[i])
        opt.step()
    return p, opt


DENSE, WHERE = ((0, 0), (0, 0)), [((0, 0), (3, 2)), ((4, 1), (0, 0)), ((1, 6), (2, 3))]


def inputs(shape, dtype):
    rng = torch.Generator().manual_seed(sum(shape))
    # networks whose gradients are of very different size: one's scale is of no use to the next
    size = 10.0 ** torch.randint(-3, 4, (shape[0],) + (1,) * (len(shape) - 1), generator=rng)
    return torch.randn(shape, generator=rng).to(dtype).cuda(), (torch.randn(shape, generator=rng) * size).to(dtype).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_dense_and_padded_populations_step_alike(evox_gpu, shape, dtype):
    p0, g0 = inputs(shape, dtype)
    p, a = steps(evox_gpu, p0, g0, DENSE, dtype)
    for where in WHERE:
        q, b = steps(evox_gpu, p0, g0, where, dtype)
        assert torch.equal(p, q)
        for name in a.state:
            assert torch.equal(a.state[name].view(torch.uint8), b.state[name].view(torch.uint8)), (where, name)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_a_checkpoint_goes_on_in_another_layout(evox_gpu, shape):
    p0, g0 = inputs(shape, torch.float32)
    p, a = steps(evox_gpu, p0, g0, DENSE, torch.float32)
    state = {name: t.clone() for name, t in a.state.items()}
    want, _ = steps(evox_gpu, p, g0, DENSE, torch.float32, 2, state)
    for where in WHERE:
        assert torch.equal(steps(evox_gpu, p, g0, where, torch.float32, 2, state)[0], want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_moments_of_each_row_by_its_own_scale(evox_gpu, shape, dtype):
    """A first step against the formula in 64 bits: the parameters, which the rounded moments have
    no part in yet, and the moments within e4m3's rounding of their own row's scales."""
    p0, g0 = inputs(shape, dtype)
    zero = torch.zeros(shape)
    want, m, v, mag, rate = adamw64(p0, g0, zero, zero, 1, HYPER["lr"], *HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
    em = 4 * U32 * mag
    bound = 3 * U32 * p0.double().cpu().abs() + rate * (em + 24 * U32 * m.abs()) + 2 * U32 * want.abs()
    r = v.sqrt()
    for where, name, x in [(where, name, x) for where in (DENSE, *WHERE) for name, x in (("m", m), ("v", r))]:
        p, opt = steps(evox_gpu, p0, g0, where, dtype, 1)
        assert ((p.double().cpu() - want).abs() <= bound + (want.abs() + bound) * U[dtype] + TINY[dtype]).all()
        got, s = held(opt, name, shape)
        # each group's scale is its own largest over 448 (roundings of the moment, of 1 / 448 and of the product)
        G, n = shape[0], math.prod(shape[1:])
        most = torch.nn.functional.pad(x.abs().reshape(G, n), (0, -n % BLOCK)).view(G, -1, BLOCK).amax(2)
        most = most.repeat_interleave(BLOCK, 1)[:, :n].reshape(shape)
        assert ((s * 448 - most).abs() <= 32 * U32 * most).all()
        # e4m3: half of 2^-3 of the number's binade, or half of 2^-9 of the scale; a root at least 2^-9 of it
        lifted = torch.where(x > 0, s * 2.0 ** -9, 0 * x) if name == "v" else 0 * x
        assert ((got - x).abs() <= x.abs() * 2.0 ** -4 + s * 2.0 ** -10 + 32 * U32 * x.abs() + lifted).all()
