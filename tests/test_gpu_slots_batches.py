"""The moves of batches: the kernels and rules that only many or large rows take (the weights'
gradient by a wave a row, both results in two passes, rows read past the caches, fewer blocks at once),
dw with dxs and without bit for bit.  Values against 64 bits at rows by chance and the last ones."""
import math

import pytest
import torch

from net_ref import DTYPES, TINY, U, U32

pytestmark = pytest.mark.gpu

F32, BF16, F16 = DTYPES


def inputs(T, k, D, dtype, aligned, weighted, seed):
    """Rows at pitches of whole lines (128 bytes) from their start, or of D + 3 from the second element; a
    tenth of the slots without a row, whose weights are NaN, and as many rows, also NaN, without a slot."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    M = T * k + 5
    pos = torch.randperm(M, generator=g, device="cuda")[:T * k].view(T, k).int()
    gone = torch.rand(T, k, generator=g, device="cuda") < 0.1
    pos[gone] = torch.tensor([-1, M, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")[torch.arange(int(gone.sum()), device="cuda") % 4]
    pos[T // 2] = -1
    there = (pos >= 0) & (pos < M)
    line = 128 // torch.finfo(dtype).bits * 8

    def rows(n):
        pitch = -(-D // line) * line if aligned else D + 3
        whole = torch.randn(n, pitch, generator=g, device="cuda").to(dtype)
        return whole[:, 0 if aligned else 1:][:, :D]

    w = None
    if weighted:
        w = torch.where(there, torch.randn(T, k, generator=g, device="cuda"), torch.full((), math.nan, device="cuda"))
    return M, pos, there, w, rows


def sample(T):
    at = torch.randperm(T, generator=torch.Generator().manual_seed(T))[:200]
    return torch.unique(torch.cat([at, torch.tensor([0, T // 2, T - 2, T - 1]).clamp_min(0)])).cuda()


def near(got, want, bound, dtype):
    got = got.double()
    limit = bound + (want.abs() + bound) * U[dtype] * 1.0001 + TINY[dtype]
    bad = ~((got - want).abs() <= limit)
    assert not bad.any(), (int(bad.sum()), got[bad][:3], want[bad][:3])


def check(evox, T, k, D, dtype, aligned=False, weighted=True):
    M, pos, there, w, rows = inputs(T, k, D, dtype, aligned, weighted, T + k + D)
    t, j = there.nonzero(as_tuple=True)
    at = pos[there].long()
    beside = lambda whole, keep: torch.equal(whole, keep)
    # dispatch
    x, xs = rows(T), rows(M)
    whole = xs._base
    keep = whole.clone()
    evox.evox_dispatch(x, pos, xs, w=w)
    want = x[t] if w is None else (w[t, j][:, None] * x[t].float()).to(dtype)  # (one product, rounded twice, as the kernel's)
    assert torch.equal(xs[at], want)
    del want
    first = xs.storage_offset()
    keep[:, first:first + D][at] = xs[at]
    assert beside(whole, keep)
    del keep
    # combine
    xs = rows(M)
    free = torch.ones(M, dtype=torch.bool, device="cuda")
    free[at] = False
    xs[free] = math.nan
    s = sample(T)
    terms = torch.where(there[s][:, :, None], xs[pos[s].long().clamp(0, M - 1)].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    W = torch.ones(len(s), k, dtype=torch.float64, device="cuda") if w is None else w[s].double().nan_to_num()
    y = evox.evox_combine(xs, pos, torch.full((T, D), 7.0, dtype=dtype, device="cuda"), w=w)
    near(y[s], (W[:, :, None] * terms).sum(1), (k + 2) * U32 * (W[:, :, None] * terms).abs().sum(1), dtype)
    assert y.isfinite().all()
    # the gradient: both, and each alone
    dy, dxs, dw = rows(T), rows(M), torch.full((T, k), 7.0, device="cuda")
    whole = dxs._base
    keep = whole.clone()
    evox.evox_combine_grad(xs, pos, dy, w=w, dxs=dxs, dw=dw)
    d = dy[s].double()[:, None, :]
    assert ((dw[s].double() - (d * terms).sum(2)).abs() <= (D + 2) * U32 * (d * terms).abs().sum(2)).all()
    assert (dw[~there] == 0).all() and dw.isfinite().all()
    want = dy[t] if w is None else (w[t, j][:, None] * dy[t].float()).to(dtype)
    assert torch.equal(dxs[at], want)
    del want
    keep[:, first:first + D][at] = dxs[at]
    assert beside(whole, keep)
    one = evox.evox_combine_grad(xs, pos, dy, w=w, dw=torch.full_like(dw, 7.0))[1]
    assert torch.equal(one, dw)
    dxs.fill_(5.0)
    keep[:, first:first + D] = 5.0
    evox.evox_combine_grad(None, pos, dy, w=w, dxs=dxs)
    keep[:, first:first + D][at] = dxs[at]
    assert beside(whole, keep)
    assert torch.equal(dxs[at], dy[t] if w is None else (w[t, j][:, None] * dy[t].float()).to(dtype))


@pytest.mark.parametrize("k", [1, 2, 4, 8, 9])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [515, 1029, 2051])
def test_weights_gradient_by_waves(evox_gpu, D, dtype, k):
    check(evox_gpu, 4097, k, D, dtype, weighted=k != 2)


# rows of which both results are in two passes: 256 lanes, four slots or more, 2^28 bytes
@pytest.mark.parametrize("T,k,D,dtype,aligned", [(16_400, 4, 2051, F16, False), (16_385, 4, 2048, BF16, True), (9_001, 5, 1500, F32, False),
                                                 (4_099, 17, 1030, F32, False), (4_096, 4, 8200, BF16, False)])
def test_both_results_in_two_passes(evox_gpu, T, k, D, dtype, aligned):
    assert T * k * D * torch.finfo(dtype).bits // 8 >= 1 << 28
    check(evox_gpu, T, k, D, dtype, aligned)


# narrow rows that start with lines and whole waves' that do not, more than the last cache holds
@pytest.mark.parametrize("T,k,D,dtype,aligned", [(262_145, 8, 64, F16, True), (300_001, 7, 64, BF16, True), (1_100_000, 2, 32, F32, True),
                                                 (33_700, 2, 1001, F32, False), (66_000, 2, 1027, F16, False), (140_000, 1, 961, BF16, False)])
def test_rows_read_past_the_caches(evox_gpu, T, k, D, dtype, aligned):
    assert T * k * D * torch.finfo(dtype).bits // 8 >= 1 << 28
    check(evox_gpu, T, k, D, dtype, aligned)


@pytest.mark.parametrize("T,k,D,dtype,aligned", [(8192, 8, 1100, BF16, False), (8200, 8, 1152, BF16, True), (8193, 5, 1029, F32, False),
                                                 (8192, 9, 1024, F32, True), (8191, 8, 1100, F16, False)])
@pytest.mark.parametrize("weighted", [False, True])
def test_many_slots_of_long_rows(evox_gpu, T, k, D, dtype, aligned, weighted):
    check(evox_gpu, T, k, D, dtype, aligned, weighted)
