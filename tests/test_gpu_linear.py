"""GPU parity of the layers of a population of networks with their definition in
64 bits.  Bounds: the textbook bound of an fp32 sum of K products in any order
and one rounding to the element type at the end; an activation (slope at most
1.13) passes the sum's error on and adds its own, taken as 4 fp32 roundings of
1 + |z|.  In 16 bits the gradient's d = dy act'(z) is rounded once before the
products: one more roundoff of the element type per term."""
import pytest
import torch

import net_ref as nr

pytestmark = pytest.mark.gpu


def layer(dtype, counts, n_in, n_out, lead=0, pad=0, shared=False, even=False, bias=True, resid=False, seed=0):
    rng = torch.Generator().manual_seed(seed)
    G, M = len(counts), sum(counts)
    xrows = M // G if shared else M
    s = {"x": nr.acts_view(rng, xrows, n_in, dtype, pad), "off": None if even or shared else nr.offsets(counts),
         "w": nr.rows_view(rng, G, n_in * n_out, dtype, lead, n_in ** -0.5).unflatten(1, (n_out, n_in)),
         "b": nr.rows_view(rng, G, n_out, dtype, lead, 0.5) if bias else None,
         "r": nr.acts_view(rng, M, n_out, dtype, pad) if resid else None,
         "z": nr.acts_view(rng, M, n_out, dtype, pad), "dy": nr.acts_view(rng, M, n_out, dtype, pad),
         "spans": nr.spans(counts), "shared": shared, "dtype": dtype}
    return s


def filled(M, n, dtype, pad=0):
    return torch.full((M, n + pad), float("nan"), dtype=dtype, device="cuda")[:, :n]


def check_forward(ev, s, act, pad=0, what="", stream=None):
    G, n_out, n_in = s["w"].shape
    M, dt = s["spans"][-1][1], s["dtype"]
    y, z = filled(M, n_out, dt, pad), filled(M, n_out, dt, pad)
    ev.evox_linear(s["x"], s["w"], y, b=s["b"], r=s["r"], z=z, off=s["off"], act=nr.ACTS.index(act), stream=stream)
    torch.cuda.synchronize()
    want_z, mag = nr.linear64(s["x"], s["w"], s["b"], s["spans"], s["shared"])
    bound = nr.sum_bound(n_in, mag)
    nr.assert_close(z, want_z, bound, dt, f"{what} z")
    want = nr.act64(want_z, act)
    bound = 1.13 * bound + (0 if act in ("none", "relu") else 4 * nr.U32 * (1 + want_z.abs()))
    if s["r"] is not None:
        want = want + s["r"].double().cpu()
        bound = bound + nr.U32 * (want.abs() + bound)
    nr.assert_close(y, want, bound, dt, f"{what} y")
    return y


def check_grad(ev, s, act, what="", pad=0):
    G, n_out, n_in = s["w"].shape
    M, dt = s["spans"][-1][1], s["dtype"]
    dx = None if s["shared"] else filled(M, n_in, dt, pad)
    dw = torch.full((G, n_out * n_in + 5), float("nan"), dtype=dt, device="cuda")
    dw_v = dw[:, 2:2 + n_out * n_in].unflatten(1, (n_out, n_in))
    db = filled(G, n_out, dt, 1)
    ev.evox_linear_grad(s["x"], s["w"], s["dy"], z=None if act == "none" else s["z"], dx=dx, dw=dw_v, db=db,
                        off=s["off"], act=nr.ACTS.index(act))
    torch.cuda.synchronize()
    x, w = s["x"].double().cpu(), s["w"].double().cpu()
    d = s["dy"].double().cpu() * nr.slope64(s["z"].double().cpu(), act)
    slope_err = 0 if act in ("none", "relu") else 8 * nr.U32 * (1 + s["z"].double().cpu().abs())
    d_err = s["dy"].double().cpu().abs() * slope_err + 2 * nr.U32 * d.abs()
    r_err = d_err + (nr.U[dt] * 1.001 if dt != torch.float32 else 0) * (d.abs() + d_err) + nr.TINY[dt]
    for g, (a, e) in enumerate(s["spans"]):
        xg = x if s["shared"] else x[a:e]
        K = e - a
        nr.assert_close(dw_v[g], d[a:e].t() @ xg,
                        nr.sum_bound(K, d[a:e].abs().t() @ xg.abs()) * 1.01 + r_err[a:e].t() @ xg.abs(), dt, f"{what} dw {g}")
        nr.assert_close(db[g], d[a:e].sum(0), (K * nr.U32 * 1.01 * d[a:e].abs() + d_err[a:e]).sum(0), dt, f"{what} db {g}")
        if dx is not None:
            nr.assert_close(dx[a:e], d[a:e] @ w[g],
                            nr.sum_bound(n_out, d[a:e].abs() @ w[g].abs()) * 1.01 + r_err[a:e] @ w[g].abs(), dt,
                            f"{what} dx {g}")


# (rows of each network, n_in, n_out): single rows, no rows, odd and tiny
# widths, fan-ins past several tiles, few and many rows
SHAPES = [([1], 1, 1), ([1] * 5, 32, 32), ([3, 0, 1, 17, 0], 17, 32), ([0, 0, 4], 7, 6), ([33] * 3, 64, 65),
          ([1, 130, 15], 129, 130), ([64, 70], 1001, 37), ([257, 3], 300, 259), ([16] * 40, 5, 3), ([700], 48, 33),
          ([2] * 3, 2500, 70), ([300, 150], 257, 264), ([9] * 20, 100, 10)]


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(evox_gpu, dtype, i):
    counts, n_in, n_out = SHAPES[i]
    act = nr.ACTS[i % 5]
    print(f"linear {dtype} {counts[:6]} {n_in}x{n_out} {act}", flush=True)
    s = layer(dtype, counts, n_in, n_out, lead=i % 4, pad=i % 3, bias=i % 4 != 3, resid=i % 2 == 0, seed=i)
    check_forward(evox_gpu, s, act, pad=i % 3, what=f"{counts[:6]} {n_in}x{n_out}")


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_gradient(evox_gpu, dtype, i):
    counts, n_in, n_out = SHAPES[i]
    act = nr.ACTS[(i + 2) % 5]
    print(f"linear_grad {dtype} {counts[:6]} {n_in}x{n_out} {act}", flush=True)
    s = layer(dtype, counts, n_in, n_out, lead=i % 4, pad=i % 3, seed=100 + i)
    check_grad(evox_gpu, s, act, f"{counts[:6]} {n_in}x{n_out}", pad=i % 3)


@pytest.mark.parametrize("act", nr.ACTS)
def test_activations(evox_gpu, act):
    s = layer(torch.float32, [40, 31], 24, 20, resid=True, seed=7)
    s["x"] = s["x"] * 6
    s["z"] = s["z"] * 4
    s["z"][0, :3] = torch.tensor([0.0, -0.0, 30.0])
    check_forward(evox_gpu, s, act)
    check_grad(evox_gpu, s, act)


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("G,n,n_in,n_out", [(7, 1, 33, 8), (12, 100, 100, 100), (3, 300, 130, 257)])
def test_shared_rows(evox_gpu, dtype, G, n, n_in, n_out):
    print(f"linear shared {dtype} {G}x{n} {n_in}x{n_out}", flush=True)
    s = layer(dtype, [n] * G, n_in, n_out, lead=1, pad=1, shared=True, seed=G)
    check_forward(evox_gpu, s, "silu", pad=1)
    check_grad(evox_gpu, s, "gelu", pad=1)


@pytest.mark.parametrize("dtype", nr.DTYPES)
def test_even_rows_and_shared_weights(evox_gpu, dtype):
    s = layer(dtype, [20] * 6, 40, 24, even=True, seed=3)
    check_forward(evox_gpu, s, "tanh")
    check_grad(evox_gpu, s, "tanh")
    s["w"] = s["w"][:1].expand(6, -1, -1)  # one W and b for all networks
    s["b"] = s["b"][:1].expand(6, -1)
    check_forward(evox_gpu, s, "tanh")


def test_rows_of_no_network_stay(evox_gpu):
    s = layer(torch.float32, [5, 6], 8, 9, seed=1)
    off = torch.tensor([2, 4, 9], dtype=torch.int32, device="cuda")
    y = torch.full((11, 9), 7.0, device="cuda")
    evox_gpu.evox_linear(s["x"], s["w"], y, off=off)
    want = torch.full((11, 9), 7.0, dtype=torch.float64)
    x, w = s["x"].double().cpu(), s["w"].double().cpu()
    want[2:4], want[4:9] = x[2:4] @ w[0].t(), x[4:9] @ w[1].t()
    assert torch.equal(y[[0, 1, 9, 10]].cpu(), want[[0, 1, 9, 10]].float())
    nr.assert_close(y, want, torch.full_like(want, 1e-5), torch.float32, "rows between")
    dx, dw, db = torch.full((11, 8), 7.0, device="cuda"), torch.empty(2, 9, 8, device="cuda"), torch.empty(2, 9, device="cuda")
    evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], dx=dx, dw=dw, db=db, off=off)
    assert (dx[[0, 1, 9, 10]] == 7.0).all()
    d = s["dy"].double().cpu()
    nr.assert_close(dw[1], d[4:9].t() @ x[4:9], torch.full((9, 8), 1e-5, dtype=torch.float64), torch.float32, "dw")
    nr.assert_close(db[0], d[2:4].sum(0), torch.full((9,), 1e-5, dtype=torch.float64), torch.float32, "db")


def test_clamped_offsets(evox_gpu):
    """Offsets past the rows, below zero or falling stay inside the buffers."""
    s = layer(torch.float32, [10, 10, 10, 10], 12, 9, seed=2)
    off = torch.tensor([-5, 12, 8, 40, 4000], dtype=torch.int32, device="cuda")
    y = torch.zeros(40, 9, device="cuda")
    evox_gpu.evox_linear(s["x"], s["w"], y, off=off)
    dx, dw, db = torch.zeros(40, 12, device="cuda"), torch.zeros(4, 9, 12, device="cuda"), torch.zeros(4, 9, device="cuda")
    evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], dx=dx, dw=dw, db=db, off=off)
    torch.cuda.synchronize()
    x, w = s["x"].double().cpu(), s["w"].double().cpu()
    nr.assert_close(y[0:8], x[0:8] @ w[0].t(), torch.full((8, 9), 1e-5, dtype=torch.float64), torch.float32, "clamped")
    assert (dw[1] == 0).all() and (dw[3] == 0).all()


@pytest.mark.parametrize("n_in,n_out,n", [(64, 48, 40), (200, 260, 150)])
def test_infinities_and_nan(evox_gpu, n_in, n_out, n):
    """A bad element shows in its own row and column, and nowhere else; the
    largest and smallest numbers keep their places."""
    s = layer(torch.float32, [n, n], n_in, n_out, seed=4)
    x, w = s["x"], s["w"]
    x[3, 5], x[7, 0], x[9] = float("inf"), float("nan"), 1e-38
    x[11, 2], x[13, 1] = 3.0e38, -float("inf")
    w[1, 6, 2] = float("nan")
    w[0, 2] = w[0, 2] * 1e30
    y = filled(2 * n, n_out, torch.float32)
    evox_gpu.evox_linear(x, w, y, off=s["off"])
    y = y.double().cpu()
    want, mag = nr.linear64(x, w, None, s["spans"], False)
    fits = want.abs() <= 3.0e38
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(y[inf], want[inf])
    ok = fits & ~torch.isnan(want)
    bound = nr.sum_bound(n_in, mag) + (n_in + 1) * 2.0 ** -126
    assert ((y - want).abs() <= bound)[ok].all()


@pytest.mark.parametrize("dtype", nr.DTYPES)
def test_reproducible_and_streams(evox_gpu, dtype):
    """The same bits on every call, on another stream, and from a graph's replays."""
    s = layer(dtype, [100, 0, 57, 300], 160, 136, lead=1, resid=True, seed=5)
    M, act = 457, evox_gpu.ACT_GELU
    y1 = check_forward(evox_gpu, s, "gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = check_forward(evox_gpu, s, "gelu", stream=side)
    assert torch.equal(y1, y2)
    out = lambda: (filled(M, 160, dtype), filled(4 * 136, 160, dtype).view(4, 136, 160), filled(4, 136, dtype))
    o1, o2, y3 = out(), out(), filled(M, 136, dtype)
    scratch = evox_gpu.evox_linear_grad_scratch(s["x"], s["w"], s["dy"])

    def both(o):
        evox_gpu.evox_linear(s["x"], s["w"], y3, b=s["b"], r=s["r"], off=s["off"], act=act)
        evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=o[0], dw=o[1], db=o[2], off=s["off"], act=act,
                                  scratch=scratch)

    both(o1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(o2)
    for _ in range(3):
        for t in (*o2, y3):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y1, y3)
        for p, q in zip(o1, o2):
            assert torch.equal(p, q)


@pytest.mark.parametrize("act", ["none", "tanh", "gelu", "silu"])
@pytest.mark.parametrize("counts,n_in,n_out", [([9, 0, 20], 12, 10), ([150, 140], 140, 150)])
def test_gradient_against_differences(evox_gpu, act, counts, n_in, n_out):
    """<gradient, direction> of L = sum c y against (L(+h) - L(-h)) / 2h, the
    sums over y in 64 bits.  Truncation: third derivatives below 2.1 times
    (h |dz|)^3 / 6 per output; rounding: the forward bound over h."""
    s = layer(torch.float32, counts, n_in, n_out, seed=6)
    M, a = sum(counts), nr.ACTS.index(act)
    rng = torch.Generator().manual_seed(8)
    c = torch.randn(M, n_out, generator=rng).cuda()
    z, y = filled(M, n_out, torch.float32), filled(M, n_out, torch.float32)
    evox_gpu.evox_linear(s["x"], s["w"], y, b=s["b"], z=z, off=s["off"], act=a)
    dx, dw, db = torch.empty_like(s["x"]), torch.empty(s["w"].shape, device="cuda"), torch.empty(s["b"].shape, device="cuda")
    evox_gpu.evox_linear_grad(s["x"], s["w"], c, z=z, dx=dx, dw=dw, db=db, off=s["off"], act=a)
    h = 2.0 ** -6
    for name, grad in (("x", dx), ("w", dw), ("b", db)):
        base = s[name]
        u = torch.randn(base.shape, generator=rng).cuda()
        L, dz = [], None
        for sign in (1, -1):
            t = dict(s, **{name: base + sign * h * u})
            evox_gpu.evox_linear(t["x"], t["w"], y, b=t["b"], off=s["off"], act=a)
            L.append(float((c.double() * y.double()).sum()))
            zt = nr.linear64(t["x"], t["w"], t["b"], s["spans"], False)[0]
            dz = zt if dz is None else dz - zt
        dz = dz.abs() / (2 * h)
        mag = nr.linear64(s["x"], s["w"], s["b"], s["spans"], False)[1]
        got, want = float((grad.double() * u.double()).sum()), (L[0] - L[1]) / (2 * h)
        cc = c.double().cpu().abs()
        trunc = float((cc * 2.1 * dz ** 3).sum()) * h * h / 6
        # roundings are of either sign: the root of the sum of squares, six times over
        per = cc * (1.13 * nr.sum_bound(n_in, 2 * mag) + 8 * nr.U32 * (1 + mag)) / h
        rounding = 6 * float(per.square().sum().sqrt()) + 1e-6 * float((grad.double().abs() * u.double().abs()).sum())
        assert abs(got - want) <= trunc + rounding, (name, got, want, trunc, rounding)


def test_long_and_wide(evox_gpu):
    """One small network with very many rows (its gradient is a sum over all of
    them), and a single row through a very wide one."""
    for counts, n_in, n_out in (([50_000], 6, 5), ([20_001, 3], 33, 20), ([1], 20_000, 3), ([1], 3, 20_000)):
        print("linear long", counts, n_in, n_out, flush=True)
        s = layer(torch.float32, counts, n_in, n_out, seed=9)
        check_forward(evox_gpu, s, "relu")
        check_grad(evox_gpu, s, "relu")
