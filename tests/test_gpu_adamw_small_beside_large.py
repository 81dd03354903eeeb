"""8-bit moments of small gradients beside a large one in their group: how far they are held off,
and what the next step makes of it."""
import pytest
import torch

from mix_ref import adamw64
from net_ref import U32

pytestmark = pytest.mark.gpu


def test_bounds_by_size(evox_gpu):
    # g from the group's largest down to 2^-27 of it, of both signs
    g = torch.exp2(-27.0 * torch.arange(256) / 255).cuda()
    g[1::2] *= -1
    p = torch.zeros(256, device="cuda")
    b1, b2, eps = 0.9, 0.99, 1e-12
    opt = evox_gpu.AdamW([p], [g], lr=1.0, betas=(b1, b2), eps=eps, weight_decay=0.0, bits=8)
    opt.step()
    s = {n: opt.state[n].double().cpu() for n in opt.state}
    m, v = (1 - b1) * g.double().cpu(), (1 - b2) ** 0.5 * g.double().cpu().abs()
    near = 16 * U32  # roundings of the moments, the ratio and the scale
    for x, name in ((m, "m"), (v, "v")):
        scale, most = s[name + "_scale"], x.abs().max()
        assert abs(scale - most / 448) <= near * most / 448
        off, normal = (s[name] * scale - x).abs(), x.abs() >= most / 28_672 * (1 + near)
        assert (off <= x.abs() * (2.0 ** -4 + near))[normal].all()
        least = x.abs() < most / 229_376 * (1 - near)
        assert least.sum() > 50
        small = ~normal & ~least if name == "v" else ~normal
        assert (off <= scale * (2.0 ** -10 + near))[small].all()
        if name == "v":
            assert (s["v"][least] == 2.0 ** -9).all()
    # the next step is the formula's of what is held: of the least ones as if their root were 2^-9 of the scale
    held_m, held_v = s["m"] * s["m_scale"], (s["v"] * s["v_scale"]) ** 2
    p.zero_()
    opt.step()
    want, m2, v2, mag, rate = adamw64(torch.zeros(256), g, held_m, held_v, 2, 1.0, b1, b2, eps, 0.0)
    assert ((p.double().cpu() - want).abs() <= rate * (4 * U32 * mag + 24 * U32 * m2.abs()) + 2 * U32 * want.abs()).all()
    assert (p.abs()[-20:] < 0.02).all() and (p.abs()[:20] > 0.8).all()
