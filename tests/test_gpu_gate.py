"""The gate and its gradient against their definitions in 64 bits."""
import math

import pytest
import torch

from mix_ref import gate64, gate_grad64, gate_weights64
from net_ref import DTYPES, TINY, U, U32

pytestmark = pytest.mark.gpu

OVER = ["chosen", "all"]


def logits(T, G, dtype, seed, pad=0, ties=False, mask=0.0):
    rng = torch.Generator().manual_seed(seed)
    z = torch.randn(T, G + pad, generator=rng) * 2
    if ties:
        z = torch.round(z)  # (with -0 among the zeros)
    z[torch.rand(T, G + pad, generator=rng) < mask] = -math.inf
    return z.to(dtype).cuda()[:, pad // 2:pad // 2 + G]


def weights_bound(z, want):
    """A weight is a quotient of an exponential (2 ulp, and its argument's rounding, times
    the argument) and a sum of as many as there are columns, each with up to three roundings
    of its exponent."""
    fine = torch.where(z.isfinite(), z, torch.zeros_like(z)).double().cpu()
    span = fine.max(1).values - fine.min(1).values
    return want.abs() * ((z.shape[1] + 16 + 4 * span) * U32)[:, None] + TINY[torch.float32]


def run(evox, z, k, over, stream=None):
    ids = torch.full((z.shape[0], k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((z.shape[0], k), math.nan, device="cuda")
    evox.evox_gate(z, ids, w, over=OVER.index(over), stream=stream)
    return ids, w


def check(z, k, over, ids, w):
    want_ids, want = gate64(z, k, over)
    assert torch.equal(ids.cpu(), want_ids), (ids.cpu() != want_ids).nonzero()[:3]
    got = w.double().cpu()
    assert torch.equal(got.isnan(), want.isnan())
    bad = ~((got - want).abs() <= weights_bound(z, want)) & ~want.isnan()
    assert not bad.any(), (got[bad][:3], want[bad][:3])


SIZES = [(1, 1, 1), (3, 2, 2), (5, 3, 1), (257, 7, 7), (9, 8, 3), (300, 31, 2), (4, 32, 32), (1, 64, 2), (65, 100, 8),
         (33, 127, 5), (10, 255, 9), (130, 256, 8), (7, 257, 16), (20, 511, 4), (20, 513, 4), (9, 1000, 32), (6, 1025, 3),
         (5, 2047, 7), (4, 2049, 8), (3, 4096, 17), (3, 5003, 2), (2, 8200, 31), (2, 16_385, 4), (2, 32_768, 32)]


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", SIZES)
def test_gate(evox_gpu, T, G, k, dtype, over):
    z = logits(T, G, dtype, T + G, pad=(G + k) % 4)
    check(z, k, over, *run(evox_gpu, z, k, over))


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", [(50, 5, 5), (40, 33, 20), (40, 100, 32), (10, 300, 32), (5, 3001, 32), (3, 12_000, 32)])
def test_ties_and_masks(evox_gpu, T, G, k, dtype, over):
    z = logits(T, G, dtype, 5 * G + k, pad=3, ties=True, mask=0.5)
    z[0] = -math.inf          # nothing left
    z[1, :] = -math.inf
    z[1, G // 2] = -3.0       # one left
    z[2, :] = 0.0             # all alike, in columns' order
    z[2, ::2] = -0.0
    check(z, k, over, *run(evox_gpu, z, k, over))


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G", [6, 70, 700, 9000])
def test_infinities_nan_and_extremes(evox_gpu, G, dtype, over):
    z = logits(8, G, dtype, G)
    z[0, 3] = math.nan
    z[1, 1], z[1, 4] = math.nan, math.nan
    z[2, 5] = math.inf
    z[3, 2], z[3, 0], z[3, 4] = math.inf, math.nan, -math.inf
    z[4, :] = torch.finfo(dtype).min    # the type's lowest is a logit like others
    z[4, 2] = -math.inf
    z[5, :] = torch.finfo(dtype).min
    z[5, 1] = torch.finfo(dtype).max
    z[6, :] = torch.finfo(dtype).tiny / 4 if dtype is not torch.float32 else 1e-40
    z[7, 1] = -math.nan
    ids, w = run(evox_gpu, z, 4, over)
    want_ids, want = gate64(z, 4, over)
    assert torch.equal(ids.cpu(), want_ids)
    got = w.double().cpu()
    assert torch.equal(got.isnan(), want.isnan())
    fine = ~want.isnan()
    # spans as large as the type's: e^-span is 0, what is left is equal logits' weights
    assert torch.allclose(got[fine], want[fine], rtol=(G + 64) * U32, atol=1e-30)


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", SIZES)
def test_gradient(evox_gpu, T, G, k, dtype, over):
    evox = evox_gpu
    z = logits(T, G, dtype, 3 * T + G, pad=(G + k) % 3, mask=0.2)
    z[T // 2] = -math.inf
    ids, w = run(evox, z, k, over)
    rng = torch.Generator().manual_seed(G)
    dw = torch.randn(T, k, generator=rng).cuda()
    dw[ids < 0] = math.nan  # of no choice: not looked at
    w[ids < 0] = math.nan
    dz = torch.full((T, G + 5), 7.0, dtype=dtype, device="cuda")
    evox.evox_gate_grad(z, ids, w, dw, dz[:, 2:2 + G], over=OVER.index(over))
    assert (dz[:, :2] == 7).all() and (dz[:, 2 + G:] == 7).all()
    want, S, mag, p = gate_grad64(z, ids, w, dw, over)
    # S: a sum of k products; a probability as in the forward; a chosen column: w (dw - S)
    es = (k + 3) * U32 * mag
    fine = torch.where(z.isfinite(), z, torch.zeros_like(z)).double().cpu()
    rel = ((G + 16 + 4 * (fine.max(1).values - fine.min(1).values)) * U32)[:, None]
    bound = p * (S.abs() * (rel + 4 * U32) + es)
    for j in range(k):
        rows = (ids[:, j] >= 0).cpu()
        at = ids[:, j].cpu().long().clamp_min(0)
        wj, dj = w[:, j].double().cpu(), dw[:, j].double().cpu()
        b = wj * (es[:, 0] + 3 * U32 * (dj.abs() + S[:, 0].abs()))
        bound[rows, at[rows]] = b[rows]
    got = dz[:, 2:2 + G].double().cpu()
    limit = bound + (want.abs() + bound) * U[dtype] + TINY[dtype]
    bad = ~((got - want).abs() <= limit)
    assert not bad.any(), (got[bad][:3], want[bad][:3], limit[bad][:3])


@pytest.mark.parametrize("over", OVER)
def test_gradient_against_differences(evox_gpu, over):
    """(w(z + h) - w(z - h)) . dw / 2h of the 64-bit gate along random directions."""
    from mix_ref import gate_weights64
    z = logits(6, 40, torch.float32, 1)
    ids, w = run(evox_gpu, z, 5, over)
    rng = torch.Generator().manual_seed(2)
    dw, dz = torch.randn(6, 5, generator=rng).cuda(), torch.empty(6, 40, device="cuda")
    evox_gpu.evox_gate_grad(z, ids, w, dw, dz, over=OVER.index(over))
    for i in range(4):
        u = torch.randn(6, 40, generator=rng).double()
        h = 1e-5
        up, down = (gate_weights64(z.cpu().double() + s * h * u, ids, over) for s in (1, -1))
        slope = ((up - down) / (2 * h) * dw.cpu().double()).sum(1)
        got = (dz.double().cpu() * u).sum(1)
        # h^2 times third derivatives of a softmax (below 10), and 64-bit roundings over h
        assert torch.allclose(got, slope, rtol=0, atol=40 * 5 * 40 * U32 + 1e-8)


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_of_the_same_choice_twice_and_of_none(evox_gpu, dtype, over):
    """A column given twice gets both slots' values, whatever the lanes' order; ids of no
    network do not count."""
    G = 24
    z = logits(3, G, dtype, 9)
    ids = torch.tensor([[4, 4, 9, -1], [1, 2, 2, 2], [G, -5, 1 << 30, 0]], dtype=torch.int32).cuda()
    w = torch.tensor([[0.25, 0.25, 0.5, 9.0], [0.25] * 4, [3.0, 4.0, 5.0, 0.5]]).cuda()
    dw = torch.tensor([[1.0, 2.0, 4.0, math.nan], [1.0, 2.0, 3.0, 4.0], [math.nan, 1.0, 2.0, 2.0]]).cuda()
    dz = [torch.empty(3, G, dtype=dtype, device="cuda") for _ in range(3)]
    for d in dz:
        evox_gpu.evox_gate_grad(z, ids, w, dw, d, over=OVER.index(over))
    assert torch.equal(dz[0], dz[1]) and torch.equal(dz[0], dz[2])
    S = [0.25 + 0.5 + 2.0, 0.25 + 0.5 + 0.75 + 1.0, 1.0]
    d = dz[0].double().cpu()
    exact = {(0, 9): 0.5 * (4 - S[0]), (1, 1): 0.25 * (1 - S[1]), (2, 0): 0.5 * (2 - S[2])}
    for (t, c), v in exact.items():
        assert d[t, c] == v
    # two slots' w dw, and each slot's own -w S
    assert d[0, 4] == 0.25 * (1 - S[0]) + 0.25 * (2 - S[0])
    assert d[1, 2] == 0.25 * (2 - S[1]) + 0.25 * (3 - S[1]) + 0.25 * (4 - S[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G", [32, 40, 333, 700, 5000])
@pytest.mark.parametrize("k", [1, 2, 3, 5, 8, 13, 16, 17, 31, 32])
def test_gradient_of_choices_by_chance(evox_gpu, k, G, dtype):
    """Rows with and without a column twice, of numbers whose sums are exact."""
    T = 77
    rng = torch.Generator().manual_seed(k + G)
    ids = torch.argsort(torch.rand(T, G, generator=rng), 1)[:, :k]
    some = torch.rand(T, k, generator=rng) < torch.tensor([0.0, 0.0, 0.1, 0.7])[torch.arange(T) % 4][:, None]
    ids = torch.where(some, ids[:, :1], ids).int()
    ids[torch.rand(T, k, generator=rng) < 0.05] = -1
    w = torch.randint(1, 5, (T, k), generator=rng) / 4
    dw = torch.randint(-4, 5, (T, k), generator=rng).float()
    z = torch.zeros(T, G, dtype=dtype, device="cuda")
    dz = torch.empty_like(z)
    evox_gpu.evox_gate_grad(z, ids.cuda(), w.cuda(), dw.cuda(), dz, over=OVER.index("chosen"))
    there = (ids >= 0).double()
    S = (w * dw * there).sum(1, keepdim=True)
    want = torch.zeros(T, G, dtype=torch.float64).scatter_add_(1, ids.clamp_min(0).long(), w * (dw - S) * there)
    assert torch.equal(dz.cpu(), want.to(dtype))


def test_empty_and_inputs_kept(evox_gpu):
    z = torch.empty(0, 9, device="cuda")
    ids, w = run(evox_gpu, z, 3, "all")
    evox_gpu.evox_gate_grad(z, ids, w, w, z)
    z = logits(70, 90, torch.bfloat16, 4)
    keep = z.clone()
    a, b = run(evox_gpu, z, 3, "all"), run(evox_gpu, z, 3, "all")
    assert torch.equal(z, keep) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_beyond_32_bits(evox_gpu, dtype):
    T, G, pitch = 70_000, 24, 65_536
    big = torch.empty(T * pitch, dtype=dtype, device="cuda").view(T, pitch)
    z = big[:, 100:100 + G]
    z.copy_(logits(T, G, dtype, 1))
    ids, w = run(evox_gpu, z, 3, "all")
    near = run(evox_gpu, z.contiguous(), 3, "all")
    assert torch.equal(ids, near[0]) and torch.equal(w, near[1])
    dw, want = torch.ones_like(w).cumsum(1), torch.empty(T, G, dtype=dtype, device="cuda")
    evox_gpu.evox_gate_grad(z.contiguous(), ids, w, dw, want, over=1)
    evox_gpu.evox_gate_grad(z, ids, w, dw, big[:, 30_000:30_000 + G], over=1)
    assert torch.equal(big[:, 30_000:30_000 + G], want)


def sorted64(z, k, over):
    """gate64 by a stable sort of all rows at once (no NaN or +inf)."""
    top, order = torch.sort(z.cpu().double() + 0.0, dim=1, descending=True, stable=True)
    ids = torch.where(top[:, :k] > -math.inf, order[:, :k], torch.full_like(order[:, :k], -1)).int()
    return ids, gate_weights64(z, ids, over)


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", [(9001, 2100, 5), (6000, 700, 32), (3001, 9001, 29), (4500, 2048, 31), (2300, 33_000 - 233, 3),
                                   (4100, 1024, 17), (20_000, 33, 33 - 1)])
def test_many_rows_and_choices(evox_gpu, T, G, k, dtype, over):
    """Batches whose rows are streamed, one wave each: ties, masks, rows in ascending and
    descending order, rows that a mask leaves little or nothing of."""
    z = logits(T, G, dtype, G + k, pad=G % 3, ties=True, mask=0.1)
    z[::5] = logits((T + 4) // 5, G, dtype, 1)
    z[1::7] = torch.sort(z[1::7], dim=1).values
    z[2::7] = torch.sort(z[2::7], dim=1, descending=True).values
    z[3::50] = -math.inf
    z[4::50, 1:] = -math.inf
    z[5::50, : G - 1] = -math.inf
    z[6::50] = torch.finfo(dtype).min
    ids, w = run(evox_gpu, z, k, over)
    want_ids, want = sorted64(z, k, over)
    assert torch.equal(ids.cpu(), want_ids)
    bound = weights_bound(z, want)
    bound[6::50] = want[6::50].abs() * (G + 64) * U32  # (equal logits: no span, but of the type's lowest value)
    bad = ~((w.double().cpu() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), w.cpu()[bad][:3], want[bad][:3])


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,G,k", [(1, 16_384, 32), (3, 8191, 9), (57, 4097, 17), (200, 16_001, 8), (256, 9000, 2), (301, 2049, 32),
                                   (1000, 5000, 12), (64, 32_768, 5), (7, 65_536 // 2 - 1, 31)])
def test_few_long_rows(evox_gpu, T, G, k, dtype, over):
    """Several waves a row: ties across their segments, masks, rows of which one wave has
    all choices or nothing."""
    z = logits(T, G, dtype, G + k, pad=G % 3, ties=True, mask=0.1)
    z[::5] = logits((T + 4) // 5, G, dtype, 1)
    z[1::7] = torch.sort(z[1::7], dim=1).values
    z[2::7] = torch.sort(z[2::7], dim=1, descending=True).values
    z[3::11] = -math.inf
    z[4::11, 1:] = -math.inf
    z[5::11, : G - 1] = -math.inf
    z[6::11, 2048:] = -math.inf
    z[0, G // 2:] = -30_000.0
    ids, w = run(evox_gpu, z, k, over)
    want_ids, want = sorted64(z, k, over)
    assert torch.equal(ids.cpu(), want_ids)
    bad = ~((w.double().cpu() - want).abs() <= weights_bound(z, want))
    assert not bad.any(), (int(bad.sum()), w.cpu()[bad][:3], want[bad][:3])
    z[0, G - 1], z[T // 2, G // 3] = math.nan, math.inf
    ids, w = run(evox_gpu, z, k, over)
    assert ids[0, 0] == G - 1 and w[0].isnan().all() and ids[T // 2, 0] == (G - 1 if T == 1 else G // 3)


@pytest.mark.parametrize("over", OVER)
@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan_among_many_rows(evox_gpu, dtype, over):
    T, G, k = 8200, 3001, 9
    z = logits(T, G, dtype, 5)
    some = torch.randperm(T, generator=torch.Generator().manual_seed(0))[:24]
    for i, t in enumerate(some.tolist()):
        z[t, (i * 131) % G] = (math.nan, math.inf, -math.nan)[i % 3]
        z[t, (i * 777 + 2100) % G] = (math.inf, math.nan, math.inf)[i % 3]
    ids, w = run(evox_gpu, z, k, over)
    want_ids, want = gate64(z[some], k, over)
    assert torch.equal(ids.cpu()[some], want_ids)
    assert torch.equal(w.cpu()[some].isnan(), want.isnan()) and want.isnan().all()
    rest = torch.ones(T, dtype=torch.bool)
    rest[some] = False
    want_ids, want = sorted64(z[rest.cuda()], k, over)
    assert torch.equal(ids.cpu()[rest], want_ids) and torch.isfinite(w.cpu()[rest]).all()
