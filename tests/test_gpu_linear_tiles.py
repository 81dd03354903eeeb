"""Every tile shape of the layers' products (forward, dx, dw; fp32, 16 bits) against
64 bits, with rows, outputs and sums that end inside a tile, a network without
rows, rows that the networks share, one W for all, and numbers that the fp32
tiles compute again.  That the sizes reach the shapes is asserted (on the host:
test_net_kernels).  Bounds as in test_gpu_linear and test_gpu_linear_grad_bits."""
import pytest
import torch

import net_ref as nr
from test_gpu_linear import filled, layer
from test_gpu_linear_grad_bits import check as check_grad_bits
from test_gpu_linear_large import check_all, close

pytestmark = pytest.mark.gpu

# networks, mean rows, n_in, n_out: between them every shape, and shares of a long sum
CASES = [(13, 210, 201, 262), (1, 2100, 201, 1001), (30, 333, 201, 391), (61, 801, 201, 262), (61, 801, 259, 262),
         (61, 333, 131, 203)]
TILES, SHARES = 16, 8
# shapes that one case each reaches with as many rows for every network: (index, [forward, dx, dw] in fp32, in 16 bits)
EVEN = {2: ([19, 18, 18], [18, 17, 17]), 3: ([17, 19, 19], [19, 19, 18])}


def ragged(G, mean):
    """Rows per network, some of them none, G mean in all."""
    u = torch.rand(G, generator=torch.Generator().manual_seed(G + mean), dtype=torch.float64)
    if G > 2:
        u[1] = u[G // 2] = 0
    counts = (u / u.sum() * G * mean).long()
    counts[-1] += G * mean - int(counts.sum())
    return counts.tolist()


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(CASES)))
def test_shapes(evox_gpu, dtype, i):
    G, mean, n_in, n_out = CASES[i]
    kernels = evox_gpu.layer_kernels(nr.DTYPES.index(dtype), G, G * mean, n_in, n_out, ragged=True)
    print(f"tiles {dtype} {CASES[i]} {kernels}", flush=True)
    s = layer(dtype, ragged(G, mean), n_in, n_out, lead=i % 3, resid=True, seed=200 + i)
    act = nr.ACTS[i % 5]
    check_all(evox_gpu, s, act, f"case {i}")
    if dtype != torch.float32 and act != "none":
        check_grad_bits(evox_gpu, s, act, f"case {i}")


def check_products(ev, s, act="none"):
    """z, y, dx, dw and db of networks with as many rows each, x shared where s says so."""
    G, n_out, n_in = s["w"].shape
    M, dt, n = s["spans"][-1][1], s["dtype"], s["spans"][0][1]
    a, x, w, b, dy = nr.ACTS.index(act), s["x"].double(), s["w"].double(), s["b"].double(), s["dy"].double()
    y, z = filled(M, n_out, dt), filled(M, n_out, dt)
    ev.evox_linear(s["x"], s["w"], y, b=s["b"], z=z, act=a)
    xs = x.expand(G, n, n_in) if s["shared"] else x.view(G, n, n_in)
    for g in range(G):
        rows = slice(g * n, (g + 1) * n)
        want = xs[g] @ w[g].t() + b[g]
        bound = nr.sum_bound(n_in, xs[g].abs() @ w[g].abs().t() + b[g].abs())
        close(z[rows], want, bound, dt, f"z {g}")
        want = nr.act64(want, act)
        close(y[rows], want, 1.13 * bound + (0 if act == "none" else 5 * nr.U32 * (1 + want.abs())), dt, f"y {g}")
    if s["w"].stride(0) == 0:
        return
    dx = None if s["shared"] else filled(M, n_in, dt)
    dw, db = filled(G * n_out, n_in, dt).view(G, n_out, n_in), filled(G, n_out, dt)
    scratch = ev.evox_linear_grad_scratch(s["x"], s["w"], s["dy"])
    scratch.fill_(255)
    ev.evox_linear_grad(s["x"], s["w"], s["dy"], dx=dx, dw=dw, db=db, scratch=scratch)
    for g in range(G):
        rows, d = slice(g * n, (g + 1) * n), dy[g * n:(g + 1) * n]
        close(dw[g], d.t() @ xs[g], nr.sum_bound(n, d.abs().t() @ xs[g].abs()), dt, f"dw {g}")
        close(db[g], d.sum(0), n * nr.U32 * 1.01 * d.abs().sum(0), dt, f"db {g}")
        if dx is not None:
            close(dx[rows], d @ w[g], nr.sum_bound(n_out, d.abs() @ w[g].abs()), dt, f"dx {g}")


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", EVEN)
@pytest.mark.parametrize("form", ["even", "shared rows", "one W"])
def test_even_and_shared(evox_gpu, dtype, i, form):
    G, n, n_in, n_out = CASES[i]
    kernels = evox_gpu.layer_kernels(nr.DTYPES.index(dtype), G, G * n, n_in, n_out)
    print(f"tiles {form} {dtype} {CASES[i]} {kernels}", flush=True)
    assert list(kernels) == EVEN[i][dtype != torch.float32]
    s = layer(dtype, [n] * G, n_in, n_out, lead=1, even=True, shared=form == "shared rows", seed=210 + i)
    if form == "one W":
        s["w"], s["b"] = s["w"][:1].expand(G, -1, -1), s["b"][:1].expand(G, -1)
    check_products(evox_gpu, s, "silu")


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", EVEN)
@pytest.mark.parametrize("where", ["x", "w", "dy"])
def test_large_numbers_infinities_and_nan(evox_gpu, dtype, i, where):
    """In fp32 also numbers too large for the split into pieces; each shows in its own
    row and column, and exact products where they are finite."""
    G, n, n_in, n_out = CASES[i]
    kernels = evox_gpu.layer_kernels(nr.DTYPES.index(dtype), G, G * n, n_in, n_out)
    print(f"tiles with bad numbers in {where} {dtype} {CASES[i]} {kernels}", flush=True)
    assert min(kernels) >= TILES
    s = layer(dtype, [n] * G, n_in, n_out, even=True, bias=False, seed=220 + i)
    t = {"x": s["x"], "w": s["w"][1], "dy": s["dy"]}[where]
    if dtype == torch.float32:
        t[3, 4], t[70, 1] = 2.0 ** 100, -1.5 * 2.0 ** 90
    t[200, 100], t[201, 7] = float("inf"), float("nan")
    y, dx = filled(G * n, n_out, dtype), filled(G * n, n_in, dtype)
    dw = filled(G * n_out, n_in, dtype).view(G, n_out, n_in)
    evox_gpu.evox_linear(s["x"], s["w"], y)
    evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], dx=dx, dw=dw)
    x, w, d = s["x"].double(), s["w"].double(), s["dy"].double()
    for g, (a, e) in enumerate(s["spans"][:4]):
        for got, p, q in ((y[a:e], x[a:e], w[g].t()), (dx[a:e], d[a:e], w[g]), (dw[g], d[a:e].t(), x[a:e])):
            want, mag = p @ q, nr.sum_bound(p.shape[1], p.abs() @ q.abs())
            got = got.double()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            inf = torch.isinf(want)
            assert torch.equal(got[inf], want[inf])
            ok = torch.isfinite(want)
            assert ((got - want).abs() <= mag + (want.abs() + mag) * nr.U[dtype] * 1.01 + nr.TINY[dtype])[ok].all()
