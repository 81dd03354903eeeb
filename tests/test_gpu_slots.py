"""Dispatch, combine and combine's gradient against their definitions in 64 bits."""
import math

import pytest
import torch

from net_ref import DTYPES, TINY, U, U32

pytestmark = pytest.mark.gpu

# (T, k, D)
SIZES = [(1, 1, 1), (1, 8, 2048), (5, 2, 3), (9, 3, 7), (300, 2, 8), (33, 4, 31), (64, 5, 64), (17, 8, 100), (301, 2, 1001),
         (7, 9, 1024), (4, 17, 2050), (3, 33, 4100), (2, 2, 8195), (40, 1, 515), (1000, 6, 16)]


def places(T, k, M, drop, seed):
    """Different rows of M for the slots, some slots with none."""
    rng = torch.Generator().manual_seed(seed)
    pos = torch.randperm(M, generator=rng)[:T * k].view(T, k).int()
    gone = torch.rand(T, k, generator=rng)
    for i, value in enumerate((-1, M, 2 ** 31 - 1, -2 ** 31)):
        pos[(gone < drop) & (gone * 97 % 4 >= i)] = value
    return pos.cuda()


def rows(M, D, dtype, seed, pad=0):
    rng = torch.Generator().manual_seed(seed)
    return torch.randn(M, D + pad, generator=rng).to(dtype).cuda()[:, pad // 2:pad // 2 + D]


def table(T, k, seed, there):
    w = torch.randn(T, k, generator=torch.Generator().manual_seed(seed)).cuda()
    return torch.where(there, w, torch.full_like(w, math.nan))  # of slots without a row: not looked at


def case(T, k, D, dtype, drop, seed):
    M, pad = T * k + 3, seed % 4
    pos = places(T, k, M, drop, seed)
    there = (pos >= 0) & (pos < M)
    return M, pad, pos, there, table(T, k, seed + 1, there)


def close(got, want, bound, dtype):
    got = got.double().cpu()
    limit = bound + (want.abs() + bound) * U[dtype] * 1.0001 + TINY[dtype]
    bad = ~((got - want).abs() <= limit)
    assert not bad.any(), (int(bad.sum()), got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("drop", [0.0, 0.4])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,k,D", SIZES)
def test_dispatch(evox_gpu, T, k, D, dtype, drop, weighted):
    M, pad, pos, there, w = case(T, k, D, dtype, drop, T + k + D)
    x = rows(T, D, dtype, D, pad)
    out = torch.full((M, D + 5), 7.0, dtype=dtype, device="cuda")
    evox_gpu.evox_dispatch(x, pos, out[:, 1:1 + D], w=w if weighted else None)
    want = torch.full((M, D + 5), 7.0, dtype=dtype)
    t, j = there.cpu().nonzero(as_tuple=True)
    m = pos.cpu()[t, j].long()
    if weighted:  # one rounding of the product, which is exact in 64 bits, to 32 bits, and one to the type
        exact = w.double().cpu()[t, j][:, None] * x.double().cpu()[t]
        close(out[:, 1:1 + D].cpu()[m], exact, exact.abs() * U32, dtype)
        want[m, 1:1 + D] = out[:, 1:1 + D].cpu()[m]
    else:
        want[m, 1:1 + D] = x.cpu()[t]
    assert torch.equal(out.cpu(), want)  # rows without a slot, and beside the rows, as they were


@pytest.mark.parametrize("weighted,residual", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("drop", [0.0, 0.4])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,k,D", SIZES)
def test_combine(evox_gpu, T, k, D, dtype, drop, weighted, residual):
    M, pad, pos, there, w = case(T, k, D, dtype, drop, T + k + D)
    pos[T // 2] = -1  # a row without any
    there[T // 2] = False
    xs, r = rows(M, D, dtype, D, pad), rows(T, D, dtype, D + 1, 3) if residual else None
    gone = torch.ones(M, dtype=torch.bool, device="cuda")
    gone[pos[there].long()] = False
    xs[gone] = math.nan  # of no slot
    y = torch.full((T, D + 3), 7.0, dtype=dtype, device="cuda")
    evox_gpu.evox_combine(xs, pos, y[:, 1:1 + D], w=w if weighted else None, r=r)
    assert (y[:, 0] == 7).all() and (y[:, 1 + D:] == 7).all()
    want, mag = torch.zeros(T, D, dtype=torch.float64), torch.zeros(T, D, dtype=torch.float64)
    for t, j in there.cpu().nonzero().tolist():
        term = (float(w[t, j]) if weighted else 1.0) * xs[pos[t, j]].double().cpu()
        want[t] += term
        mag[t] += term.abs()
    if residual:
        want += r.double().cpu()
        mag += r.double().cpu().abs()
    close(y[:, 1:1 + D], want, (k + 2) * U32 * mag, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,k,D", SIZES + [(3000, 2, 1029), (2000, 3, 2051), (500, 1, 9001)])
def test_residual_in_the_result_s_place(evox_gpu, T, k, D, dtype):
    M, pad, pos, there, w = case(T, k, D, dtype, 0.2, T + k + D)
    xs, r = rows(M, D, dtype, D, pad), rows(T, D, dtype, D + 1, 3)
    want = evox_gpu.evox_combine(xs, pos, torch.empty(T, D, dtype=dtype, device="cuda"), w=w, r=r)
    whole = r._base.clone()
    got = evox_gpu.evox_combine(xs, pos, r, w=w, r=r)
    assert torch.equal(got, want)
    assert torch.equal(r._base[:, :1], whole[:, :1]) and torch.equal(r._base[:, 1 + D:], whole[:, 1 + D:])


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("drop", [0.0, 0.4])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,k,D", SIZES)
def test_combine_gradient(evox_gpu, T, k, D, dtype, drop, weighted):
    M, pad, pos, there, w = case(T, k, D, dtype, drop, T + k + D)
    xs, dy = rows(M, D, dtype, D, pad), rows(T, D, dtype, D + 1, 3)
    gone = torch.ones(M, dtype=torch.bool, device="cuda")
    gone[pos[there].long()] = False
    xs[gone] = math.nan
    dxs, dw = torch.full((M, D + 2), 7.0, dtype=dtype, device="cuda"), torch.full((T, k), 7.0, device="cuda")
    call = lambda **kw: evox_gpu.evox_combine_grad(xs, pos, dy, w=w if weighted else None, **kw)
    call(dxs=dxs[:, 1:1 + D], dw=dw)
    want = torch.full((M, D + 2), 7.0, dtype=dtype)
    t, j = there.cpu().nonzero(as_tuple=True)
    m = pos.cpu()[t, j].long()
    d = dy.double().cpu()[t]
    exact = d * (w.double().cpu()[t, j][:, None] if weighted else 1.0)
    close(dxs[:, 1:1 + D].cpu()[m], exact, exact.abs() * U32, dtype)
    want[m, 1:1 + D] = dxs[:, 1:1 + D].cpu()[m]
    assert torch.equal(dxs.cpu(), want)
    slope, mag = torch.zeros(T, k, dtype=torch.float64), torch.zeros(T, k, dtype=torch.float64)
    slope[t, j] = (d * xs.double().cpu()[m]).sum(1)
    mag[t, j] = (d * xs.double().cpu()[m]).abs().sum(1)
    assert ((dw.double().cpu() - slope).abs() <= (D + 2) * U32 * mag).all()
    # each by itself, the same bits
    only, one = torch.full_like(dxs, 7.0), torch.full_like(dw, 7.0)
    call(dw=one)
    evox_gpu.evox_combine_grad(None, pos, dy, w=w if weighted else None, dxs=only[:, 1:1 + D])
    assert torch.equal(one, dw) and torch.equal(only, dxs)
    # and in place
    if pad == 0:
        call(dxs=xs)
        assert torch.equal(xs[m.cuda()], dxs[:, 1:1 + D][m.cuda()])


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_of_a_weighted_dispatch_against_differences(evox_gpu, dtype):
    """<g, dispatch(x, w)> is linear in x and in w: differences of the 64-bit form are exact."""
    evox, (T, k, D) = evox_gpu, (20, 3, 50)
    M, _, pos, there, w = case(T, k, D, dtype, 0.3, 8)
    x, g = rows(T, D, dtype, 1), rows(M, D, dtype, 2)
    dx, dw = torch.empty(T, D, dtype=dtype, device="cuda"), torch.empty(T, k, device="cuda")
    evox.evox_combine(g, pos, dx, w=w)
    evox.evox_combine_grad(g, pos, x, dw=dw)
    W = torch.where(there, w, torch.zeros_like(w)).double().cpu()
    at, X, Gd = pos.cpu().long().clamp(0, M - 1), x.double().cpu(), g.double().cpu()
    f = lambda X, W: (W[:, :, None] * Gd[at] * X[:, None, :] * there.cpu()[:, :, None]).sum()
    rng = torch.Generator().manual_seed(3)
    for _ in range(3):
        u, h = torch.randn(T, D, generator=rng).double(), torch.randn(T, k, generator=rng).double()
        slope = f(X + u, W) - f(X, W)
        got = (dx.double().cpu() * u).sum()
        assert abs(got - slope) <= (u.abs() * (dx.double().cpu().abs() * U[dtype] * 2 + k * U32 * 40)).sum() + 1e-9
        slope = f(X, W + h) - f(X, W)
        mag = (Gd[at].abs() * X.abs()[:, None, :]).sum(2)
        assert abs((dw.double().cpu() * h).sum() - slope) <= (h.abs() * mag).sum() * (D + 2) * U32 + 1e-9


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_beyond_32_bits(evox_gpu, dtype):
    evox, (T, k, D, pitch) = evox_gpu, (6, 2, 40, 60_000)
    M = 80_000
    big = torch.empty(M * pitch, dtype=dtype, device="cuda").view(M, pitch)
    pos = torch.tensor([[M - 1, 0], [M - 2, 77_777], [1, 72_000], [60_000, 2], [-1, M - 3], [M, 3]], dtype=torch.int32).cuda()
    x, w = rows(T, D, dtype, 1), torch.full((T, k), 0.5, device="cuda")
    xs = big[:, 50:50 + D]
    evox.evox_dispatch(x, pos, xs, w=w)
    t, j = ((pos >= 0) & (pos < M)).nonzero(as_tuple=True)
    assert torch.equal(xs[pos[t, j].long()], x[t] * 0.5)
    y, dw = torch.empty(T, D, dtype=dtype, device="cuda"), torch.empty(T, k, device="cuda")
    evox.evox_combine(xs, pos, y)
    count = torch.zeros(T, device="cuda").index_add_(0, t, torch.ones(len(t), device="cuda"))
    assert torch.equal(y, x * (0.5 * count)[:, None].to(dtype))
    evox.evox_combine_grad(xs, pos, y, dxs=xs)
    assert torch.equal(xs[pos[t, j].long()], y[t])


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_in_rows(evox_gpu, dtype):
    """They reach their own rows' results alone; weight 0 times infinity is NaN, as it is."""
    evox = evox_gpu
    pos = torch.tensor([[0, 1], [2, 3], [-1, 4]], dtype=torch.int32).cuda()
    xs = rows(6, 20, dtype, 3)
    xs[0, 5], xs[2, 6], xs[5] = math.inf, math.nan, math.nan
    w = torch.tensor([[0.0, 1.0], [1.0, 1.0], [math.inf, 1.0]]).cuda()
    y = torch.empty(3, 20, dtype=dtype, device="cuda")
    evox.evox_combine(xs, pos, y, w=w)
    bad = torch.zeros(3, 20, dtype=torch.bool, device="cuda")
    bad[0, 5] = bad[1, 6] = True
    assert torch.equal(y.isnan(), bad) and torch.equal(y[2], xs[4])


def test_nothing_to_do(evox_gpu):
    evox = evox_gpu
    new = lambda *s, d=torch.float32: torch.zeros(*s, dtype=d, device="cuda")
    pos = new(0, 2, d=torch.int32)
    evox.evox_dispatch(new(0, 5), pos, new(0, 5))
    evox.evox_combine(new(0, 5), pos, new(0, 5))
    evox.evox_combine_grad(new(0, 5), pos, new(0, 5), dxs=new(0, 5), dw=new(0, 2))
    # no rows of the networks: every slot has none
    pos, y, dw = new(3, 2, d=torch.int32), new(3, 5) + 7, new(3, 2) + 7
    evox.evox_dispatch(new(3, 5), pos, new(0, 5))
    evox.evox_combine(new(0, 5), pos, y, r=new(3, 5) + 2)
    evox.evox_combine_grad(new(0, 5), pos, new(3, 5), dw=dw)
    assert (y == 2).all() and (dw == 0).all()
