"""The optimizer's step against its formula in 64 bits."""
import math

import pytest
import torch

from mix_ref import adamw64
from net_ref import DTYPES, TINY, U, U32

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, DECAY = 3e-3, 0.9, 0.99, 1e-6, 0.05
HYPER = dict(lr=LR, betas=(B1, B2), eps=EPS, weight_decay=DECAY)

# shapes of the tensors of a step; "rows": views of the rows of one wider matrix
LISTS = {
    "one": [(1,)], "small": [(7,), (3, 5), (2, 3, 4)], "block": [(255,), (256,), (257,), (512,), (1000,)],
    "rows": [(5, 3), (5, 4, 8), (5, 300), (5, 1)], "many rows": [(300, 17), (300, 33), (300, 130)],
    "wide rows": [(3, 1001), (3, 2050)], "large": [(1001, 1003), (70_000,)], "many": [(n % 13 + 1, n % 29 + 1) for n in range(100)],
    "empty": [(0,), (4, 5), (3, 0), (0, 7)], "all empty": [(0,)],
}


def tensors(kind, dtype, seed):
    """(whole, views) of parameters or gradients."""
    rng = torch.Generator().manual_seed(seed)
    shapes = LISTS[kind]
    if "rows" not in kind:
        out = [torch.randn(*s, generator=rng).to(dtype).cuda() for s in shapes]
        return out, out
    width = sum(math.prod(s[1:]) + 1 for s in shapes) + seed % 5
    X = torch.randn(shapes[0][0], width, generator=rng).to(dtype).cuda()
    views, at = [], 1
    for s in shapes:
        n = math.prod(s[1:])
        views.append(X[:, at:at + n].view(s) if len(s) == 2 else X[:, at:at + n].unflatten(1, s[1:]))
        at += n + 1
    return [X], views


class Held:
    """The states of an optimizer by tensor, as the 64-bit numbers that they stand for."""

    def __init__(self, opt, bits):
        self.m, self.v, self.scales, self.master = [], [], [], []
        at, block = 0, 0
        for i, p in enumerate(opt.params):
            rows, n = opt._shapes[i][:2]
            N, per = rows * n, -(-n // 256)
            for name, out in (("m", self.m), ("v", self.v)):
                x = opt.state[name][at:at + N].double().cpu().view(rows, n)
                if bits == 8:
                    s = opt.state[name + "_scale"][block:block + rows * per].double().cpu().view(rows, per)
                    x = x * s.repeat_interleave(256, 1)[:, :n]
                    if name == "m":
                        self.scales.append(s.repeat_interleave(256, 1)[:, :n].reshape(p.shape))
                    else:
                        self.scales[-1] = (self.scales[-1], s.repeat_interleave(256, 1)[:, :n].reshape(p.shape))
                out.append(x.reshape(p.shape))
            if "master" in opt.state:
                self.master.append(opt.state["master"][at:at + N].double().cpu().reshape(p.shape))
            at, block = at + N, block + rows * per


def within(got, want, bound, what):
    bad = ~((got.double().cpu() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), got.cpu()[bad][:3], want[bad][:3], bound[bad][:3])


def check(opt, before, p0, g, bits, dtype, t):
    after = Held(opt, bits)
    for i, p in enumerate(opt.params):
        old_p = before.master[i] if before.master else p0[i].double().cpu()
        old_v = before.v[i] ** 2 if bits == 8 else before.v[i]
        want, m, v, mag, rate = adamw64(old_p, g[i], before.m[i], old_v, t, LR, B1, B2, EPS, DECAY)
        # every operation rounds once to 32 bits, and so do the constants: m is two products
        # and a sum, v one product more (and of 8 bits a square of a product), the step a
        # quotient whose parts have a handful of roundings, the decay a product and two sums
        em, ev = 4 * U32 * mag, 8 * U32 * v
        bound = 3 * U32 * old_p.abs() + rate * (em + 24 * U32 * m.abs()) + 2 * U32 * want.abs()
        low = TINY[torch.float32]
        if before.master:
            within(after.master[i], want, bound + low, "master")
        within(p, want, bound + (want.abs() + bound) * U[dtype] + TINY[dtype], "p")
        if bits == 32:
            within(after.m[i], m, em + low, "m")
            within(after.v[i], v, ev + low, "v")
            continue
        # e4m3: half of 2^-3 of the number's binade, or of 2^-9 of the scale; the root at
        # least 2^-9 of it where it is not 0.  Held: number times scale, each once rounded.
        sm, sv = after.scales[i]
        r = v.sqrt()
        within(after.m[i], m, m.abs() * 2.0 ** -4 + sm * 2.0 ** -10 + em * 2 + 16 * U32 * m.abs() + 2.0 ** -100, "m")
        within(after.v[i], r, r * 2.0 ** -4 + sv * 2.0 ** -10 + 16 * U32 * r + torch.where(r > 0, sv * 2.0 ** -9, 0 * r) + low, "v")
        assert ((after.v[i] > 0) == (r > 2.0 ** -75)).all()
        # the group's largest is held by the scale to its roundings
    return after


@pytest.mark.parametrize("kind", sorted(LISTS))
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", DTYPES)
def test_steps(evox_gpu, kind, bits, dtype, master):
    if master and dtype is torch.float32:
        with pytest.raises(evox_gpu.EvoxError):
            evox_gpu.AdamW(*[[torch.zeros(3, device="cuda")] for _ in range(2)], master=True)
        return
    whole, params = tensors(kind, dtype, 3)
    gwhole, grads = tensors(kind, dtype, 8)
    opt = evox_gpu.AdamW(params, grads, bits=bits, master=master, **HYPER)
    before = Held(opt, bits)
    for t in range(1, 4):
        for w in gwhole:
            w.mul_(-0.5 if t == 2 else 1.25)
        p0, beside = [p.clone() for p in params], [w.clone() for w in whole]
        opt.step()
        assert opt.state["t"].item() == t
        before = check(opt, before, p0, grads, bits, dtype, t)
        for p, q in zip(params, p0):  # what lies beside the parameters is as it was
            p_now = p.clone()
            p.copy_(q)
            q.copy_(p_now)
        assert all(torch.equal(w, b) for w, b in zip(whole, beside))
        for p, q in zip(params, p0):
            p.copy_(q)


@pytest.mark.parametrize("bits", [32, 8])
def test_strided_gradients_of_dense_parameters(evox_gpu, bits):
    p = torch.randn(6, 300, device="cuda")
    g = torch.randn(6, 310, device="cuda")[:, 4:304]
    q, h = p.clone(), g.contiguous()
    a, b = evox_gpu.AdamW([p], [g], bits=bits, **HYPER), evox_gpu.AdamW([q.view(6, 300)], [h], bits=bits, **HYPER)
    a.step()
    b.step()
    if bits == 32:
        assert torch.equal(p, q) and torch.equal(a.state["v"], b.state["v"])
    before = Held(evox_gpu.AdamW([q], [g], bits=bits), bits)
    assert a.state["m"].numel() == 1800 and before.m[0].shape == (6, 300)


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_go_on_counting(evox_gpu, bits):
    """A replayed graph is the same as as many eager steps, the learning rate read from the
    device."""
    evox = evox_gpu
    torch.manual_seed(0)
    start = [torch.randn(200, 33, device="cuda"), torch.randn(5000, device="cuda")]
    grads = [torch.randn_like(p) for p in start]
    runs = []
    for _ in range(2):
        params, lr = [p.clone() for p in start], torch.tensor([1e-2], device="cuda")
        runs.append((params, lr, evox.AdamW(params, grads, lr=lr, bits=bits)))
    (pa, la, a), (pb, lb, b) = runs
    a.step()
    b.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for i in range(4):
        la.mul_(0.5)
        lb.mul_(0.5)
        for g in grads:
            g.add_(0.1)
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert a.state["t"].item() == b.state["t"].item() == i + 2
        assert all(torch.equal(x, y) for x, y in zip(pa, pb))
        for name in a.state:
            assert torch.equal(a.state[name].view(torch.uint8), b.state[name].view(torch.uint8)), name


def test_rate_as_number_and_on_the_device_and_many_steps(evox_gpu):
    """And the count's powers far on: at step 10^6 the corrections are 1."""
    p, g = torch.randn(1000, device="cuda"), torch.randn(1000, device="cuda")
    runs = []
    for lr in (1e-2, torch.tensor([1e-2], device="cuda")):
        q = p.clone()
        opt = evox_gpu.AdamW([q], [g], lr=lr, betas=(B1, B2), eps=EPS, weight_decay=DECAY)
        opt.state["t"].fill_(999_999)
        opt.state["m"].copy_(g * 0.5)
        opt.state["v"].copy_(g * g)
        opt.step()
        runs.append(q)
    want, m, v, mag, rate = adamw64(p, g, g.double() * 0.5, g.double() ** 2, 10 ** 6, 1e-2, B1, B2, EPS, DECAY)
    for q in runs:  # (1e-2 as fp32 is 2^-25 of itself away)
        assert ((q.double().cpu() - want).abs() <= 4 * U32 * p.abs().double().cpu() + rate * 40 * U32 * mag).all()


@pytest.mark.parametrize("n", [1024, 1021, 5])
@pytest.mark.parametrize("bits", [32, 8])
def test_infinities_and_nan(evox_gpu, bits, n):
    """They stay in their own elements, step after step; the others are as without them."""
    torch.manual_seed(1)
    start, g = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    odd = torch.zeros(n, dtype=torch.bool, device="cuda")
    odd[[3] if n < 300 else [3, 300]] = True
    g[600:700] = 0.0
    runs = []
    for bad in (False, True):
        p, d = start.clone(), g.clone()
        d[odd] = 0.0  # (without them: nothing in these elements)
        if bad:
            d[3] = math.nan
            if n > 300:
                d[300] = math.inf
        opt = evox_gpu.AdamW([p], [d], bits=bits)
        opt.step()
        d.masked_fill_(odd, 0.0)  # one such gradient, then none
        opt.step()
        runs.append((p, opt.state))
    (p, a), (q, b) = runs
    assert torch.equal(q.isnan(), odd) and torch.equal(p[~odd], q[~odd])
    for name in "mv":
        x, y = a[name].float(), b[name].float()
        assert torch.equal(x[~odd], y[~odd]) and not torch.isfinite(y[odd]).any()
        if bits == 8:
            assert torch.equal(a[name + "_scale"], b[name + "_scale"])


def test_8_bits_hold_every_e4m3_number(evox_gpu):
    """m = 0.1 g of a first step: a group whose numbers are multiples of its largest over
    448 by e4m3 numbers is held exactly."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    q = torch.where(codes.isnan(), torch.zeros_like(codes), codes)
    g = q.cuda() * 2.0 ** -6
    p = torch.zeros(256, device="cuda")
    opt = evox_gpu.AdamW([p], [g], bits=8)
    opt.step()
    assert torch.equal(opt.state["m"].float().cpu(), q)
    # the roots |g| sqrt(1 - b2) are in the same proportions, above 0 at least 2^-9
    assert torch.equal(opt.state["v"].float().cpu(), q.abs())


@pytest.mark.parametrize("bits", [32, 8])
def test_load(evox_gpu, bits):
    evox = evox_gpu
    g = torch.randn(700, device="cuda")
    p = [torch.randn(700, device="cuda")]
    a = evox.AdamW(p, [g], bits=bits)
    a.step()
    q = [p[0].clone()]
    b = evox.AdamW(q, [g], bits=bits)
    b.load({k: v.clone() for k, v in a.state.items()})
    a.step()
    b.step()
    assert torch.equal(p[0], q[0]) and b.state["t"].item() == 2
    with pytest.raises(evox.EvoxError):
        b.load({"t": a.state["t"]})
    with pytest.raises(evox.EvoxError):
        b.load(dict(a.state, m=a.state["m"][:5]))


def test_offsets_beyond_32_bits(evox_gpu):
    """More than 2^31 elements, in bytes beyond 2^32: the last ones are where they belong."""
    n = (1 << 31) + 4099
    p = torch.full((n,), 1.0, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 5000, (1 << 31) - 1, 1 << 31, n - 4097, n - 260, n - 3, n - 1], device="cuda")
    g[at] = 2.0
    opt = evox_gpu.AdamW([p], [g], lr=0.25, weight_decay=0.0, bits=8)
    opt.step()
    assert (p[at] == 0.75).all() and int((p != 1.0).sum()) == len(at)
    assert int((opt.state["m"].view(torch.uint8) != 0).sum()) == len(at)
    held = opt.state["m"][at].float() * opt.state["m_scale"][at // 256]
    assert ((held - 0.2).abs() <= 0.2 * 2.0 ** -4).all()


def test_rates_of_zero_and_below(evox_gpu):
    """A rate of 0 leaves the parameters and moves the states; a negative one ascends."""
    p, g = torch.randn(700, device="cuda"), torch.randn(700, device="cuda")
    g[:100] = 0.0
    for bits in (32, 8):
        q = p.clone()
        opt = evox_gpu.AdamW([q], [g], lr=0.0, bits=bits)
        opt.step()
        assert torch.equal(q, p) and opt.state["t"].item() == 1 and (opt.state["m"].float() != 0).any()
        up, down = p.clone(), p.clone()
        for t, lr in ((up, -1e-2), (down, 1e-2)):
            evox_gpu.AdamW([t], [g], lr=lr, weight_decay=0.0, bits=bits).step()
        # (two roundings of p each)
        assert ((up + down - 2 * p).abs() <= 8 * U32 * (p.abs() + 1)).all() and ((up - p) * g >= 0).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr,eps", [(1.0, 1e-40), (1e3, 1e-36), (-1.0, 1e-42), (1e-3, 1e-30)])
def test_eps_next_to_nothing(evox_gpu, bits, lr, eps):
    """A gradient of 0 changes nothing, whatever divides it; the others move by the rate, m / sqrt(v)
    being 1 at the first step (of 8 roundings)."""
    g = torch.randn(700, device="cuda")
    g[g.abs() < 0.1] = 0.0
    p = torch.zeros(700, device="cuda")
    evox_gpu.AdamW([p], [g], lr=lr, eps=eps, weight_decay=0.0, bits=bits).step()
    assert ((p + lr * g.sign()).abs() <= 16 * U32 * abs(lr)).all()
