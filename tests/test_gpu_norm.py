"""GPU parity of the layer norm and of the cross-entropy fitness of a population
of networks with their definitions in 64 bits.  Bounds: fp32 sums of D terms
(in any order) and one rounding to the element type."""
import math

import pytest
import torch

import net_ref as nr

pytestmark = pytest.mark.gpu
EPS = 1e-5
# (rows of each network, row length)
SHAPES = [([1], 1), ([1] * 9, 2), ([3, 0, 70, 0], 17), ([5] * 40, 32), ([33, 1], 100), ([0, 200], 129), ([600], 64),
          ([40, 41], 1001), ([7, 3], 1024), ([2, 9], 4099), ([3], 32768), ([1, 4], 20_001), ([150, 0, 31], 513)]


def filled(M, n, dtype, pad=0):
    return torch.full((M, n + pad), float("nan"), dtype=dtype, device="cuda")[:, :n]


def norm_inputs(dtype, counts, D, pad=0, lead=0, seed=0, even=False):
    rng = torch.Generator().manual_seed(seed)
    G, M = len(counts), sum(counts)
    P = nr.rows_view(rng, G, 2 * D, dtype, lead, 0.5)
    return {"x": (nr.acts_view(rng, M, D + pad, dtype) * 1.5 + 0.75)[:, :D], "gamma": P[:, :D],
            "beta": P[:, D:], "dy": nr.acts_view(rng, M, D, dtype, pad), "off": None if even else nr.offsets(counts),
            "spans": nr.spans(counts), "dtype": dtype, "D": D, "M": M, "G": G}


def stats64(x):
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    return mean, rstd


def per_row(s, p):
    p = p.double().cpu()
    return torch.cat([p[g:g + 1].expand(e - a, -1) for g, (a, e) in enumerate(s["spans"])])


def check_norm(ev, s, pad=0, stream=None):
    M, D, dt = s["M"], s["D"], s["dtype"]
    y, mean, rstd = filled(M, D, dt, pad), filled(M, 1, torch.float32).view(-1), filled(M, 1, torch.float32).view(-1)
    ev.evox_layernorm(s["x"], s["gamma"], s["beta"], y, mean=mean, rstd=rstd, off=s["off"], eps=EPS, stream=stream)
    torch.cuda.synchronize()
    x = s["x"].double().cpu()
    m, r = stats64(x)
    # the mean's error, the centred elements', the variance's, rstd's
    e_mean = (D + 2) * nr.U32 * x.abs().mean(1, keepdim=True)
    e_c = e_mean + nr.U32 * (x - m).abs()
    e_r = r * ((D + 6) * nr.U32 + e_mean * r + 2 * (e_mean * r) ** 2)
    nr.assert_close(mean, m[:, 0], e_mean[:, 0], torch.float32, "mean")
    nr.assert_close(rstd, r[:, 0], e_r[:, 0], torch.float32, "rstd")
    gamma, beta = per_row(s, s["gamma"]), per_row(s, s["beta"])
    want = (x - m) * r * gamma + beta
    bound = (e_c * r + (x - m).abs() * e_r) * gamma.abs() * 1.01 + 4 * nr.U32 * (want.abs() + beta.abs())
    nr.assert_close(y, want, bound, dt, "y")
    return y, mean, rstd


def check_norm_grad(ev, s, pad=0):
    M, D, G, dt = s["M"], s["D"], s["G"], s["dtype"]
    x, dy = s["x"].double().cpu(), s["dy"].double().cpu()
    m, r = stats64(x)
    mean, rstd = m[:, 0].float().cuda(), r[:, 0].float().cuda()
    m, r = mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
    dx, dg, db = filled(M, D, dt, pad), filled(G, D, dt, pad), filled(G, D, dt, pad)
    ev.evox_layernorm_grad(s["x"], s["gamma"], mean, rstd, s["dy"], dx, dg, db, off=s["off"])
    torch.cuda.synchronize()
    gamma = per_row(s, s["gamma"])
    h, a = (x - m) * r, dy * gamma
    e_h = 3 * nr.U32 * (h.abs() + m.abs() * r)
    m1, m2 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    want = r * (a - m1 - h * m2)
    e1 = (D + 3) * nr.U32 * a.abs().mean(1, keepdim=True)
    e2 = (D + 4) * nr.U32 * (a * h).abs().mean(1, keepdim=True) + (a.abs() * e_h).mean(1, keepdim=True)
    bound = r * (e1 + h.abs() * e2 + e_h * m2.abs() + 6 * nr.U32 * (a.abs() + m1.abs() + (h * m2).abs())) * 1.01
    nr.assert_close(dx, want, bound, dt, "dx")
    for g, (a0, e) in enumerate(s["spans"]):
        n, t = e - a0, dy[a0:e] * h[a0:e]
        nr.assert_close(db[g], dy[a0:e].sum(0), n * nr.U32 * 1.01 * dy[a0:e].abs().sum(0), dt, f"dbeta {g}")
        nr.assert_close(dg[g], t.sum(0), (n + 2) * nr.U32 * 1.01 * t.abs().sum(0) + (dy[a0:e].abs() * e_h[a0:e]).sum(0),
                        dt, f"dgamma {g}")
    return dx, dg, db


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_layernorm(evox_gpu, dtype, i):
    counts, D = SHAPES[i]
    print(f"layernorm {dtype} {counts[:6]} {D}", flush=True)
    s = norm_inputs(dtype, counts, D, pad=i % 3, lead=i % 4, seed=i)
    check_norm(evox_gpu, s, pad=i % 3)


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_layernorm_gradient(evox_gpu, dtype, i):
    counts, D = SHAPES[i]
    print(f"layernorm_grad {dtype} {counts[:6]} {D}", flush=True)
    s = norm_inputs(dtype, counts, D, pad=i % 3, lead=i % 4, seed=50 + i)
    check_norm_grad(evox_gpu, s, pad=i % 3)


def test_layernorm_even_shared_and_long(evox_gpu):
    s = norm_inputs(torch.float32, [8] * 12, 50, seed=1, even=True)
    check_norm(evox_gpu, s)
    check_norm_grad(evox_gpu, s)
    s["gamma"], s["beta"] = s["gamma"][:1].expand(12, -1), s["beta"][:1].expand(12, -1)
    check_norm(evox_gpu, s)
    s = norm_inputs(torch.float32, [30_000, 0, 11], 40, seed=2)
    check_norm(evox_gpu, s)
    check_norm_grad(evox_gpu, s)


def test_layernorm_constant_and_bad_rows(evox_gpu):
    s = norm_inputs(torch.float32, [6], 300, seed=3)
    s["x"][0] = 4.0
    s["x"][1, 7] = float("nan")
    s["x"][2, 7] = float("inf")
    y = filled(6, 300, torch.float32)
    evox_gpu.evox_layernorm(s["x"], s["gamma"], s["beta"], y, eps=EPS)
    assert torch.equal(y[0], s["beta"][0])
    assert torch.isnan(y[1:3]).all() and torch.isfinite(y[3:]).all()


def test_norm_in_place_streams_and_graph(evox_gpu):
    s = norm_inputs(torch.bfloat16, [70, 0, 300], 260, seed=4)
    y, mean, rstd = check_norm(evox_gpu, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(check_norm(evox_gpu, s, stream=side)[0], y)
    dx, dg, db = check_norm_grad(evox_gpu, s)
    scratch = evox_gpu.evox_layernorm_grad_scratch(s["x"], s["gamma"])
    x64 = s["x"].double().cpu()
    m, r = stats64(x64)
    mean, rstd = m[:, 0].float().cuda(), r[:, 0].float().cuda()
    buf, dg2, db2 = s["dy"].clone(), torch.empty_like(dg), torch.empty_like(db)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # dx in the place of dy
        evox_gpu.evox_layernorm_grad(s["x"], s["gamma"], mean, rstd, buf, buf, dg2, db2, off=s["off"], scratch=scratch)
    for _ in range(3):
        buf.copy_(s["dy"])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buf, dx) and torch.equal(dg2, dg) and torch.equal(db2, db)


def test_norm_gradient_against_differences(evox_gpu):
    """Central differences of L = sum c y in x, gamma and beta (sums over y in 64
    bits): truncation of the order h^2 (here 2^-12 of the gradient's terms),
    rounding of the order 2^-24 / h per output."""
    counts, D = [9, 0, 30], 70
    s = norm_inputs(torch.float32, counts, D, seed=5)
    M = s["M"]
    rng = torch.Generator().manual_seed(6)
    c = torch.randn(M, D, generator=rng).cuda()
    y, mean, rstd = check_norm(evox_gpu, s)
    dx, dg, db = filled(M, D, torch.float32), filled(3, D, torch.float32), filled(3, D, torch.float32)
    evox_gpu.evox_layernorm_grad(s["x"], s["gamma"], mean, rstd, c, dx, dg, db, off=s["off"])
    h = 2.0 ** -7
    P = torch.cat([s["gamma"], s["beta"]], 1)
    for name, grad in (("x", dx), ("p", torch.cat([dg, db], 1))):
        u = torch.randn(grad.shape, generator=rng).cuda()
        L = []
        for sign in (1, -1):
            x = s["x"] + sign * h * u if name == "x" else s["x"]
            p = P + sign * h * u if name == "p" else P
            evox_gpu.evox_layernorm(x, p[:, :D], p[:, D:], y, off=s["off"], eps=EPS)
            L.append(float((c.double() * y.double()).sum()))
        got, want = float((grad.double() * u.double()).sum()), (L[0] - L[1]) / (2 * h)
        terms = float((grad.double() * u.double()).square().sum().sqrt())
        limit = 2.0 ** -11 * terms * math.sqrt(M) + 12 * 2.0 ** -22 / h * float(c.double().norm())
        assert abs(got - want) <= limit, (name, got, want, limit)


# ---------------------------------------------------------------------------
XSHAPES = [([1], 1), ([1] * 7, 2), ([3, 9, 70, 2], 10), ([32] * 50, 10), ([33, 1], 100), ([5, 200], 129), ([600], 3),
           ([40, 41], 1001), ([7, 3], 1024), ([2, 9], 4099), ([3], 32768), ([1, 4], 20_001)]


def xent_inputs(dtype, counts, C, pad=0, seed=0, shared=False, ignore=0.1):
    rng = torch.Generator().manual_seed(seed)
    G, M = len(counts), sum(counts)
    rows = M // G if shared else M
    lab = torch.randint(0, C, (rows,), generator=rng, dtype=torch.int32)
    bad = torch.rand(rows, generator=rng) < ignore
    lab[bad] = torch.where(torch.rand(int(bad.sum()), generator=rng) < 0.5, -1, C).int()
    return {"z": nr.acts_view(rng, M, C, dtype, pad, 3.0), "labels": lab.cuda(), "G": G, "M": M, "C": C, "dtype": dtype,
            "off": None if shared else nr.offsets(counts), "spans": nr.spans(counts), "shared": shared}


def check_xent(ev, s, pad=0, grad=True):
    M, C, G, dt = s["M"], s["C"], s["G"], s["dtype"]
    fit, dz = filled(G, 1, torch.float32).view(-1), filled(M, C, dt, pad)
    ev.evox_xent(s["z"], s["labels"], fit, dz=dz if grad else None, off=s["off"])
    torch.cuda.synchronize()
    z, lab = s["z"].double().cpu(), s["labels"].long().cpu()
    for g, (a, e) in enumerate(s["spans"]):
        lg = lab if s["shared"] else lab[a:e]
        ok = (lg >= 0) & (lg < C)
        n = int(ok.sum())
        logp = torch.log_softmax(z[a:e], 1)
        if n == 0:
            assert math.isnan(float(fit[g]))
            assert not grad or (dz[a:e] == 0).all()
            continue
        want = -logp[ok].gather(1, lg[ok][:, None]).mean()
        spread = (z[a:e].max(1).values - z[a:e].min(1).values)[ok].max()
        # exp to 2 units and of an argument rounded once, a sum of C of them, its log
        e_p = (C + 4) * nr.U32 + spread * nr.U32
        nr.assert_close(fit[g:g + 1], want[None], torch.tensor([e_p + 4 * nr.U32 * (1 + spread + math.log(C))]),
                        torch.float32, f"fit {g}")
        if grad:
            hot = torch.zeros(e - a, C, dtype=torch.float64)
            hot[ok] = hot[ok].scatter(1, lg[ok][:, None], 1.0)
            d = (logp.exp() - hot) * ok[:, None] / n
            nr.assert_close(dz[a:e], d, (logp.exp() * (e_p + 4 * nr.U32) + hot * 4 * nr.U32) / n * ok[:, None], dt, f"dz {g}")
    return fit, dz


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(XSHAPES)))
def test_xent(evox_gpu, dtype, i):
    counts, C = XSHAPES[i]
    print(f"xent {dtype} {counts[:6]} {C}", flush=True)
    s = xent_inputs(dtype, counts, C, pad=i % 3, seed=i, ignore=0.0 if max(counts) < 4 else 0.1)
    f1, dz = check_xent(evox_gpu, s, pad=i % 3)
    f2, _ = check_xent(evox_gpu, s, grad=False)
    assert torch.equal(f1, f2) or torch.isnan(f1).any()
    z = s["z"]
    if z.stride(0) == dz.stride(0) or z.shape[0] == 1:  # the gradient in the logits' place
        fit = torch.empty_like(f1)
        evox_gpu.evox_xent(z, s["labels"], fit, dz=z, off=s["off"])
        assert torch.equal(z, dz)


@pytest.mark.parametrize("G,n,C", [(5, 1, 3), (300, 32, 10), (4, 100, 1000)])
def test_xent_shared_labels(evox_gpu, G, n, C):
    check_xent(evox_gpu, xent_inputs(torch.float32, [n] * G, C, shared=True, seed=G))


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("C", [6, 700, 9000])
def test_xent_left_out_classes(evox_gpu, dtype, C):
    """-inf and the type's lowest value as masks; rows that they leave empty,
    networks without a row or without a label."""
    s = xent_inputs(dtype, [4, 0, 3, 2], C, seed=C, ignore=0.0)
    z, lab = s["z"], s["labels"]
    low = torch.finfo(dtype).min
    lab[:] = C - 1
    lab[7:] = -1
    z[0, :C - 1] = -float("inf")          # only the label's class is left: loss 0
    z[1, : C // 2] = low
    z[2, : C // 2] = -float("inf")
    z[3] = low                            # all the same: log C
    z[4] = -float("inf")                  # nothing left
    z[5, C - 1] = -float("inf")           # the label's class is left out
    fit, dz = torch.empty(4, device="cuda"), filled(9, C, dtype)
    evox_gpu.evox_xent(z, lab, fit, dz=dz, off=s["off"])
    zz = z.double().cpu()
    logp = torch.log_softmax(zz[:4], 1)
    want = -logp[:, C - 1].mean()
    assert abs(float(fit[0]) - float(want)) <= 1e-5 * (1 + abs(float(want)))
    d = logp.exp()
    d[:, C - 1] -= 1
    nr.assert_close(dz[:4], d / 4, (C + 30) * nr.U32 * (d.abs() + 1e-3), dtype, "masked dz")
    assert math.isnan(float(fit[1])) and math.isnan(float(fit[2])) and math.isnan(float(fit[3]))
    assert torch.isnan(dz[4]).all()
    assert float(dz[5, C - 1].float()) == pytest.approx(-1 / 3, rel=2e-2)
    assert (dz[7:] == 0).all()
    one = torch.empty(1, device="cuda")
    evox_gpu.evox_xent(z[5:6].contiguous(), lab[5:6].contiguous(), one)
    assert float(one) == math.inf


def test_xent_against_differences(evox_gpu):
    s = xent_inputs(torch.float32, [20, 11], 30, seed=11)
    fit, dz = check_xent(evox_gpu, s)
    rng = torch.Generator().manual_seed(12)
    u = torch.randn(31, 30, generator=rng).cuda()
    h = 2.0 ** -6
    L = []
    for sign in (1, -1):
        f = torch.empty(2, device="cuda")
        evox_gpu.evox_xent(s["z"] + sign * h * u, s["labels"], f, off=s["off"])
        L.append(float(f.double().sum()))
    got, want = float((dz.double() * u.double()).sum()), (L[0] - L[1]) / (2 * h)
    # third derivatives of log-sum-exp are below 2 |u|^3 per row; fitness rounding 2^-23 / h
    limit = 2 * float(u.abs().max()) ** 3 * 2 * h * h / 6 + 8 * 2.0 ** -23 * 8 / h
    assert abs(got - want) <= limit, (got, want, limit)


def test_xent_graph_and_repeat(evox_gpu):
    s = xent_inputs(torch.bfloat16, [300, 17, 64], 500, seed=13)
    fit, dz = check_xent(evox_gpu, s)
    scratch = evox_gpu.evox_xent_scratch(s["z"], fit)
    f2, d2 = torch.empty_like(fit), torch.empty_like(dz)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        evox_gpu.evox_xent(s["z"], s["labels"], f2, dz=d2, off=s["off"], scratch=scratch)
    for _ in range(3):
        f2.fill_(0)
        d2.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(f2, fit) and torch.equal(d2, dz)


def test_rows_of_no_network_stay(evox_gpu):
    off = torch.tensor([2, 2, 5], dtype=torch.int32, device="cuda")
    x = torch.randn(7, 20, device="cuda")
    p = torch.ones(2, 20, device="cuda")
    y = torch.full((7, 20), 3.0, device="cuda")
    evox_gpu.evox_layernorm(x, p, p, y, off=off)
    assert (y[[0, 1, 5, 6]] == 3.0).all() and not (y[2:5] == 3.0).all()
    dx = torch.full((7, 20), 3.0, device="cuda")
    stat = torch.ones(7, device="cuda")
    dg, db = torch.empty(2, 20, device="cuda"), torch.empty(2, 20, device="cuda")
    evox_gpu.evox_layernorm_grad(x, p, stat, stat, y, dx, dg, db, off=off)
    assert (dx[[0, 1, 5, 6]] == 3.0).all() and (dg[0] == 0).all() and (db[0] == 0).all()
    dz, fit = torch.full((7, 20), 3.0, device="cuda"), torch.empty(2, device="cuda")
    evox_gpu.evox_xent(x, torch.zeros(7, dtype=torch.int32, device="cuda"), fit, dz=dz, off=off)
    assert (dz[[0, 1, 5, 6]] == 3.0).all() and math.isnan(float(fit[0])) and math.isfinite(float(fit[1]))
