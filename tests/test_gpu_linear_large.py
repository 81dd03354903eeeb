"""The layers' larger tiles, shares of a long sum, pitches that pass 32 bits and
scratch contents, against 64 bits on the GPU.  Bounds as in test_gpu_linear."""
import pytest
import torch

import net_ref as nr
from test_gpu_linear import filled, layer

pytestmark = pytest.mark.gpu


def close(got, want, bound, dtype, what):
    got = got.double()
    limit = bound + (want.abs() + bound) * nr.U[dtype] * 1.0001 + nr.TINY[dtype]
    bad = ~((got - want).abs() <= limit)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, e.g. {got[bad][:3].tolist()} for {want[bad][:3].tolist()}"


def check_all(ev, s, act, what):
    """Forward with the residual in y's place, and the gradient, from a scratch full of NaN."""
    G, n_out, n_in = s["w"].shape
    M, dt, a = s["spans"][-1][1], s["dtype"], nr.ACTS.index(act)
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    y, z = s["r"].clone(), filled(M, n_out, dt)
    ev.evox_linear(s["x"], s["w"], y, b=s["b"], r=y, z=z, off=s["off"], act=a)
    dx, dw, db = filled(M, n_in, dt), filled(G * n_out, n_in, dt).view(G, n_out, n_in), filled(G, n_out, dt)
    scratch = ev.evox_linear_grad_scratch(s["x"], s["w"], s["dy"])
    scratch.fill_(255)
    ev.evox_linear_grad(s["x"], s["w"], s["dy"], z=None if act == "none" else s["z"], dx=dx, dw=dw, db=db, off=s["off"],
                        act=a, scratch=scratch)
    torch.cuda.synchronize()
    zz = s["z"].double()
    d = s["dy"].double() * nr.slope64(zz, act)
    d_err = s["dy"].double().abs() * (0 if act in ("none", "relu") else 8 * nr.U32 * (1 + zz.abs())) + 2 * nr.U32 * d.abs()
    r_err = d_err + (nr.U[dt] * 1.001 if dt != torch.float32 else 0) * (d.abs() + d_err) + nr.TINY[dt]
    for g, (lo, hi) in enumerate(s["spans"]):
        xg, dg = x[lo:hi], d[lo:hi]
        want = xg @ w[g].t() + b[g]
        bound = nr.sum_bound(n_in, xg.abs() @ w[g].abs().t() + b[g].abs())
        close(z[lo:hi], want, bound, dt, f"{what} z {g}")
        want = nr.act64(want, act)
        bound = 1.13 * bound + (0 if act in ("none", "relu") else 4 * nr.U32 * (1 + want.abs()) * 1.2)
        res = s["r"][lo:hi].double()
        close(y[lo:hi], want + res, bound + nr.U32 * (want + res).abs(), dt, f"{what} y {g}")
        K = hi - lo
        close(dw[g], dg.t() @ xg, nr.sum_bound(K, dg.abs().t() @ xg.abs()) * 1.01 + r_err[lo:hi].t() @ xg.abs(), dt, f"{what} dw {g}")
        close(db[g], dg.sum(0), (K * nr.U32 * 1.01 * dg.abs() + d_err[lo:hi]).sum(0), dt, f"{what} db {g}")
        close(dx[lo:hi], dg @ w[g], nr.sum_bound(n_out, dg.abs() @ w[g].abs()) * 1.01 + r_err[lo:hi] @ w[g].abs(), dt, f"{what} dx {g}")


# rows that fill and overrun the tiles of every shape, K that ends inside one; few
# tiles with long sums (in dx: fan-out, in dw: rows)
CASES = [([600, 0, 257, 1, 900] * 3, 190, 777, "gelu"), ([256] * 12, 512, 512, "none"), ([130] * 100, 96, 300, "relu"),
         ([300, 500], 520, 1030, "silu"), ([40, 25], 70, 3000, "tanh"), ([9000], 70, 130, "gelu"),
         ([5000, 0, 2100], 8, 190, "relu"), ([3] * 40, 300, 5, "silu"), ([2] * 9, 1000, 600, "none")]


@pytest.mark.parametrize("dtype", nr.DTYPES)
@pytest.mark.parametrize("i", range(len(CASES)))
def test_large(evox_gpu, dtype, i):
    counts, n_in, n_out, act = CASES[i]
    print(f"large {dtype} {counts[:5]} x{len(counts)} {n_in}x{n_out} {act}", flush=True)
    check_all(evox_gpu, layer(dtype, counts, n_in, n_out, lead=i % 3, resid=True, seed=20 + i), act, f"case {i}")


@pytest.mark.parametrize("where", ["x", "w", "dy"])
def test_large_numbers_in_tiles(evox_gpu, where):
    """Numbers too large for the split into bf16 pieces, an infinity and a NaN, in
    tiles through LDS (fp32): exact products where they are finite."""
    s = layer(torch.float32, [300, 280], 260, 270, seed=30)
    t = {"x": s["x"], "w": s["w"][1], "dy": s["dy"]}[where]
    t[3, 4], t[70, 1] = 2.0 ** 100, -1.5 * 2.0 ** 90
    t[200, 100], t[201, 7] = float("inf"), float("nan")
    y = filled(580, 270, torch.float32)
    dx, dw = filled(580, 260, torch.float32), filled(540, 260, torch.float32).view(2, 270, 260)
    evox_gpu.evox_linear(s["x"], s["w"], y, off=s["off"])
    evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], dx=dx, dw=dw, off=s["off"])
    x, w, d = s["x"].double(), s["w"].double(), s["dy"].double()
    for g, (a, e) in enumerate(s["spans"]):
        for got, p, q in ((y[a:e], x[a:e], w[g].t()), (dx[a:e], d[a:e], w[g]), (dw[g], d[a:e].t(), x[a:e])):
            want, mag = p @ q, nr.sum_bound(p.shape[1], p.abs() @ q.abs())
            got = got.double()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            inf = torch.isinf(want)
            assert torch.equal(got[inf], want[inf])
            ok = torch.isfinite(want)
            assert ((got - want).abs() <= mag + want.abs() * nr.U32 * 1.01)[ok].all()


@pytest.mark.parametrize("n_in,n_out", [(40, 24), (130, 100)])
def test_pitches_past_32_bits(evox_gpu, n_in, n_out):
    """Rows whose offsets pass 2^31 elements (and 2^32 bytes)."""
    M, ld, dt = 66_000, 32_800, torch.bfloat16
    assert M * ld > 2 ** 31
    buf = torch.empty(M * ld, dtype=dt, device="cuda").view(M, ld)
    s = layer(dt, [M // 2, M // 2], n_in, n_out, even=True, seed=31)
    x, y, dx = buf[:, :n_in], buf[:, 200:200 + n_out], buf[:, 400:400 + n_in]
    x.copy_(s["x"])
    evox_gpu.evox_linear(x, s["w"], y, b=s["b"], act=evox_gpu.ACT_RELU)
    evox_gpu.evox_linear_grad(x, s["w"], y, dx=dx)
    yy, dd = filled(M, n_out, dt), filled(M, n_in, dt)
    evox_gpu.evox_linear(s["x"], s["w"], yy, b=s["b"], act=evox_gpu.ACT_RELU)
    evox_gpu.evox_linear_grad(s["x"], s["w"], yy, dx=dd)
    assert torch.equal(y, yy) and torch.equal(dx, dd)


def test_norm_and_loss_scratch_and_pitches(evox_gpu):
    """The norm's and the loss's results do not depend on what the scratch holds, nor
    on pitches past 32 bits."""
    M, D, ld = 66_000, 100, 32_800
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = torch.randn(M, D, generator=g, device="cuda"), torch.randn(M, D, generator=g, device="cuda")
    gamma = torch.randn(3, D, generator=g, device="cuda")
    off = torch.tensor([0, 20_000, 20_001, M], dtype=torch.int32, device="cuda")
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    outs = []
    big = torch.empty(M * ld, device="cuda").view(M, ld)
    for fill, wide in ((0, False), (255, False), (255, True)):
        put = (lambda t, at: big[:, at:at + D].copy_(t)) if wide else (lambda t, at: t)
        new = (lambda at: big[:, at:at + D]) if wide else (lambda at: torch.empty(M, D, device="cuda"))
        xx, dd, y, dx, dz = put(x, 0), put(dy, 100), new(200), new(300), new(400)
        evox_gpu.evox_layernorm(xx, gamma, gamma, y, mean=mean, rstd=rstd, off=off)
        dg, db, fit = torch.empty(3, D, device="cuda"), torch.empty(3, D, device="cuda"), torch.empty(3, device="cuda")
        s1 = evox_gpu.evox_layernorm_grad_scratch(xx, gamma)
        s2 = evox_gpu.evox_xent_scratch(xx, fit)
        s1.fill_(fill)
        s2.fill_(fill)
        evox_gpu.evox_layernorm_grad(xx, gamma, mean, rstd, dd, dx, dg, db, off=off, scratch=s1)
        labels = torch.arange(M, device="cuda", dtype=torch.int32) % (D + 7) - 3
        evox_gpu.evox_xent(xx, labels, fit, dz=dz, off=off, scratch=s2)
        outs.append([t.clone() for t in (y, dx, dg, db, fit, dz)])
    for other in outs[1:]:
        assert all(torch.equal(p, q) for p, q in zip(outs[0], other))
