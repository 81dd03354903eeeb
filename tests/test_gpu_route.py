"""Slots sorted by network against a list per network."""
import pytest
import torch

from mix_ref import route64

pytestmark = pytest.mark.gpu


def choices(T, k, G, kind, seed):
    rng = torch.Generator().manual_seed(seed)
    if kind == "one":
        ids = torch.full((T, k), G // 2)
    elif kind == "none":
        ids = torch.full((T, k), -1)
    elif kind == "few":
        ids = (torch.rand(T, k, generator=rng) ** 4 * G).long().clamp_max(G - 1)
    else:
        ids = torch.randint(0, G, (T, k), generator=rng)
        gone = torch.rand(T, k, generator=rng)
        for share, value in ((0.05, -1), (0.03, G), (0.02, 2 ** 31 - 1), (0.01, -2 ** 31)):
            ids[gone < share] = value
    return ids.int().cuda()


def run(evox, ids, G, src=True, scratch=None, stream=None):
    n = ids.numel()
    off = torch.full((G + 1,), -9, dtype=torch.int32, device="cuda")
    pos = torch.full(tuple(ids.shape), -9, dtype=torch.int32, device="cuda")
    back = torch.full((n,), -9, dtype=torch.int32, device="cuda") if src else None
    evox.evox_route(ids, off, pos, src=back, scratch=scratch, stream=stream)
    return off, pos, back


def check(ids, G, off, pos, back):
    want_off, want_pos, want_src = route64(ids, G)
    assert torch.equal(off.cpu(), want_off)
    assert torch.equal(pos.cpu(), want_pos)
    if back is not None:
        n = len(want_src)
        assert back[:n].cpu().tolist() == want_src and (back[n:] == -9).all()  # the rest as it was


SLOTS = [(1, 1), (1, 8), (9, 7), (64, 1), (13, 5), (255, 1), (128, 2), (257, 1), (1024, 1), (205, 5), (2048, 1), (683, 3), (4095, 1), (512, 8), (4097, 1), (1366, 6),
         (8192, 8), (16_384, 2), (32_769, 1), (10_007, 2), (65_537, 1), (25_000, 8)]


@pytest.mark.parametrize("kind", ["mixed", "few", "one", "none"])
@pytest.mark.parametrize("G", [1, 2, 3, 64, 100, 1000, 2048])
@pytest.mark.parametrize("T,k", SLOTS)
def test_route(evox_gpu, T, k, G, kind):
    ids = choices(T, k, G, kind, T + k + G)
    check(ids, G, *run(evox_gpu, ids, G))


@pytest.mark.parametrize("kind", ["mixed", "few", "one", "none"])
@pytest.mark.parametrize("G", [2049, 4097, 32_768, 32_769, 70_000, 1 << 20])
@pytest.mark.parametrize("T,k", [(1, 8), (1, 1), (63, 1), (700, 3), (4096, 1), (4097, 1), (30_000, 2), (100_003, 1)])
def test_many_networks(evox_gpu, T, k, G, kind):
    ids = choices(T, k, G, kind, T + k + G)
    check(ids, G, *run(evox_gpu, ids, G))


def test_without_src_and_empty(evox_gpu):
    ids = choices(300, 3, 10, "mixed", 1)
    check(ids, 10, *run(evox_gpu, ids, 10, src=False))
    ids = torch.empty(0, 4, dtype=torch.int32, device="cuda")
    off, _, _ = run(evox_gpu, ids, 5)
    assert off.tolist() == [0] * 6
    off, _, _ = run(evox_gpu, ids, 5000)
    assert off.tolist() == [0] * 5001


def test_large(evox_gpu):
    """More slots than the tests against lists take, by their properties: a permutation,
    networks in order, slots in order within one."""
    T, k, G = 1_000_003, 4, 600
    ids = choices(T, k, G, "mixed", 3)
    off, pos, back = run(evox_gpu, ids, G)
    flat, n = ids.flatten().long(), int(off[-1])
    kept = (flat >= 0) & (flat < G)
    assert n == int(kept.sum()) and torch.equal(pos.flatten() >= 0, kept)
    src = back[:n].long()
    assert torch.equal(pos.flatten()[src], torch.arange(n, device="cuda", dtype=torch.int32))
    key = flat[src] * (T * k) + src
    assert (key[1:] > key[:-1]).all()
    assert torch.equal(off.long(), torch.searchsorted(flat[src], torch.arange(G + 1, device="cuda")))


def test_graph_with_shared_scratch(evox_gpu):
    """Two captured sorts that share their scratch, replayed in turn with other ids."""
    evox = evox_gpu
    calls = []
    for T, G in ((20_000, 300), (9000, 3000)):
        ids = choices(T, 2, G, "mixed", G)
        calls.append((ids, G, [torch.empty(G + 1, dtype=torch.int32, device="cuda"), torch.empty_like(ids),
                               torch.full((2 * T,), -9, dtype=torch.int32, device="cuda")]))
    scratch = torch.empty(max(evox.evox_route_scratch(c[0], c[2][0]).numel() for c in calls), dtype=torch.uint8, device="cuda")
    graphs = []
    for ids, G, (off, pos, back) in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            evox.evox_route(ids, off, pos, src=back, scratch=scratch)
        graphs.append(g)
    for turn in range(3):
        for g, (ids, G, out) in zip(graphs, calls):
            ids.copy_(choices(ids.shape[0], 2, G, "mixed" if turn else "few", 10 * turn + G))
            out[2].fill_(-9)
            g.replay()
            check(ids, G, *out)
