"""The e4m3 numbers of 8-bit moments are those of the formula in 64 bits, but for numbers that
fp32's roundings may move over the middle between two of them; and the same bits each time."""
import pytest
import torch

from net_ref import DTYPES, U32

pytestmark = pytest.mark.gpu

B1, B2 = 0.9, 0.999


def nearest(q):
    """e4m3 numbers nearest to q, ties to the even one."""
    unit = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(q / unit) * unit


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(4096, 1024), (3000, 700), (100_000, 9)])
def test_codes(evox_gpu, shape, dtype):
    G, n = shape
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda: torch.randn(shape, generator=g, device="cuda")
    p, d = normal().to(dtype), (normal() * 0.02).to(dtype)
    runs = []
    for _ in range(2):
        opt = evox_gpu.AdamW([p.clone()], [d], betas=(B1, B2), bits=8)
        s = opt.state
        at = torch.Generator(device="cuda").manual_seed(1)
        for name in ("m", "v"):
            codes = torch.randint(0, 127 if name == "v" else 254, s[name].shape, generator=at, device="cuda")
            codes += (codes > 126).long()  # (0x7f is NaN)
            s[name].view(torch.uint8).copy_(codes)
            s[name + "_scale"].copy_(torch.rand(s[name + "_scale"].shape, generator=at, device="cuda") * 1e-4)
        s["t"].fill_(1000)
        spread = lambda x: x.double().view(G, -1).repeat_interleave(256, 1)[:, :n]
        old = {name: s[name].double().view(G, n) * spread(s[name + "_scale"]) for name in ("m", "v")}
        opt.step()
        runs.append({name: t.clone() for name, t in s.items()})
    assert all(torch.equal(runs[0][name].view(torch.uint8), runs[1][name].view(torch.uint8)) for name in s)
    x = d.double()
    terms = (B1 * old["m"]).abs() + (1 - B1) * x.abs()
    # the products' and the sum's roundings and the constants' (6 of fp32), of the terms; of v 8, of
    # which its root has half, and the root 2 of its own
    new = {"m": (B1 * old["m"] + (1 - B1) * x, 6 * U32 * terms), "v": ((B2 * old["v"] ** 2 + (1 - B2) * x * x).sqrt(), None)}
    new["v"] = (new["v"][0], 6 * U32 * new["v"][0])
    for name, (want, off) in new.items():
        pad = torch.nn.functional.pad(want.abs(), (0, -n % 256)).view(G, -1, 256)
        most = pad.amax(2).repeat_interleave(256, 1)[:, :n]
        off_most = torch.nn.functional.pad(off, (0, -n % 256)).view(G, -1, 256).amax(2).repeat_interleave(256, 1)[:, :n]
        q = want * (448 / most)
        # the number's own error, the largest one's, and roundings of the ratio and of the product
        room = off * (448 / most) + q.abs() * (off_most / most + 4 * U32)
        low, high = (torch.sign(q) * nearest((q.abs() + r).clamp(0, 448)) for r in (-room, room))
        got = runs[0][name].double().view(G, n)
        if name == "v":
            low, high = (torch.where((t == 0) & (q > 0), 2.0 ** -9, t) for t in (low, high))
        bad = ~((got == low) | (got == high) | (q.abs() <= room) & (got == 0))
        assert not bad.any(), (name, int(bad.sum()), got[bad][:3], q[bad][:3])
        assert int((low != high).sum()) <= q.numel() * 2e-3  # (the room decides next to nothing)
        exact = nearest(q)
        if name == "v":
            exact = torch.where((q > 0) & (exact == 0), 2.0 ** -9, exact)
        assert int((got != exact).sum()) <= q.numel() * 2e-5
