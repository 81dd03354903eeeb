"""The gradient of 16-bit layers against 64 bits with one rounding, that of the
results: what lies between, d = dy act'(z), keeps at least twice the type's bits
and a wider range, whichever kernels a size takes.

Bounds: |d - kept d| <= u^2 |d| (two numbers of unit roundoff u), plus 2^-34 in
f16 (whose smallest number is 2^-24: the second one is kept 2^10 times larger);
the slope's own error as in test_gpu_linear; an fp32 sum of 2 K products."""
import pytest
import torch

import net_ref as nr
from test_gpu_linear import filled, layer
from test_gpu_linear_large import close

pytestmark = pytest.mark.gpu


def check(ev, s, act, what, bias=True):
    G, n_out, n_in = s["w"].shape
    M, dt = s["spans"][-1][1], s["dtype"]
    dx, dw = filled(M, n_in, dt), filled(G * n_out, n_in, dt).view(G, n_out, n_in)
    db = filled(G, n_out, dt) if bias else None
    scratch = ev.evox_linear_grad_scratch(s["x"], s["w"], s["dy"])
    scratch.fill_(255)
    ev.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=dx, dw=dw, db=db, off=s["off"], act=nr.ACTS.index(act),
                        scratch=scratch)
    torch.cuda.synchronize()
    x, w, zz, dy = (s[k].double() for k in ("x", "w", "z", "dy"))
    d = dy * nr.slope64(zz, act)
    d_err = dy.abs() * (0 if act == "relu" else 8 * nr.U32 * (1 + zz.abs())) + 2 * nr.U32 * d.abs()
    kept = d_err + nr.U[dt] ** 2 * 1.01 * (d.abs() + d_err) + (2.0 ** -34 if dt == torch.float16 else 2.0 ** -126)
    for g, (lo, hi) in enumerate(s["spans"]):
        xg, dg, K = x[lo:hi], d[lo:hi], hi - lo
        close(dw[g], dg.t() @ xg, nr.sum_bound(2 * K, dg.abs().t() @ xg.abs()) * 1.01 + kept[lo:hi].t() @ xg.abs(), dt,
              f"{what} dw {g}")
        if bias:
            close(db[g], dg.sum(0), (K * nr.U32 * 1.01 * dg.abs() + d_err[lo:hi]).sum(0), dt, f"{what} db {g}")
        close(dx[lo:hi], dg @ w[g], nr.sum_bound(2 * n_out, dg.abs() @ w[g].abs()) * 1.01 + kept[lo:hi] @ w[g].abs(), dt,
              f"{what} dx {g}")


# narrow, few inputs, tiles of every shape, shares of a long sum (in dx, in dw), short sums (of dx, of dw)
CASES = [([300, 0, 41], 40, 33), ([64, 70], 20, 300), ([130, 0, 257, 1], 190, 300), ([600, 500, 100] * 6, 515, 530),
         ([40, 25], 70, 3000), ([9000], 70, 130), ([50, 3] * 10, 300, 5), ([2, 0, 3] * 9, 200, 100)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["relu", "tanh", "gelu", "silu"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_one_rounding(evox_gpu, dtype, act, i):
    counts, n_in, n_out = CASES[i]
    print(f"gradient bits {dtype} {counts[:4]} x{len(counts)} {n_in}x{n_out} {act}", flush=True)
    check(evox_gpu, layer(dtype, counts, n_in, n_out, lead=i % 2, seed=80 + i), act, f"case {i} {act}")


@pytest.mark.parametrize("i", range(len(CASES)))
def test_range_of_f16(evox_gpu, i):
    """dy at both ends of f16's range: d above the largest number (a slope may be
    1.13) and below the smallest normal one, in results that are well inside it (but
    for the large d's sum)."""
    counts, n_in, n_out = CASES[i]
    print(f"gradient range {counts[:4]} x{len(counts)} {n_in}x{n_out}", flush=True)
    for scale, back in ((2.0 ** -17, 2.0 ** 9), (2.0 ** 14, 2.0 ** -11)):
        s = layer(torch.float16, counts, n_in, n_out, seed=90 + i)
        s["dy"] = (s["dy"] * scale).clamp(-65504, 65504)
        if scale > 1:
            s["dy"][::7, ::3], s["z"][::7, ::3] = 65504.0, 1.5
        s["x"], s["w"] = s["x"] * back, s["w"] * (back * n_in ** 0.5 / 8)
        check(evox_gpu, s, "gelu", f"case {i} scale {scale}", bias=scale < 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n_in,n_out,n", [(200, 260, 150), (20, 300, 70)])
def test_infinities_and_nan_in_dy(evox_gpu, dtype, n_in, n_out, n):
    """An infinite or NaN element of dy shows in its own row and column as in 64
    bits, and nowhere else."""
    s = layer(dtype, [n, n], n_in, n_out, seed=95)
    s["dy"][3, 5], s["dy"][7, 6], s["dy"][n + 9, 8] = float("inf"), float("nan"), -float("inf")
    dx, dw = filled(2 * n, n_in, dtype), filled(2 * n_out, n_in, dtype).view(2, n_out, n_in)
    evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=dx, dw=dw, off=s["off"], act=evox_gpu.ACT_GELU)
    d = s["dy"].double() * nr.slope64(s["z"].double(), "gelu")
    for g, (a, e) in enumerate(s["spans"]):
        for got, want in ((dx[a:e], d[a:e] @ s["w"][g].double()), (dw[g], d[a:e].t() @ s["x"][a:e].double())):
            got = got.double()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            inf = torch.isinf(want)
            assert torch.equal(got[inf], want[inf]) and inf.any()


# few rows per network (both of d's numbers in one tile of dx): rows past one such
# tile, none, odd widths, shares of a long fan-out
PAIRS = [([9, 0, 32, 1, 70, 33, 2] * 3, 200, 260), ([32] * 20, 64, 128), ([12, 5, 20], 331, 1756), ([1] * 50, 130, 90),
         ([5, 31] * 9, 515, 67), ([20], 49, 50)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["relu", "tanh", "gelu", "silu"])
@pytest.mark.parametrize("i", range(len(PAIRS)))
def test_one_rounding_of_few_rows(evox_gpu, dtype, act, i):
    counts, n_in, n_out = PAIRS[i]
    print(f"gradient bits {dtype} {counts[:4]} x{len(counts)} {n_in}x{n_out} {act}", flush=True)
    check(evox_gpu, layer(dtype, counts, n_in, n_out, lead=i % 2, even=len(set(counts)) == 1, seed=110 + i), act, f"case {i} {act}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_rows_leave_the_others(evox_gpu, dtype):
    """Rows of no network stay, and offsets past the rows stay inside the buffers."""
    s = layer(dtype, [10, 10, 10, 10], 130, 90, seed=120)
    for off, mine in (([2, 4, 4, 30, 35], [(2, 4, 0), (4, 30, 2), (30, 35, 3)]), ([-5, 12, 8, 40, 4000], [(0, 8, 0), (12, 40, 2)])):
        dx = torch.full((40, 130), 7.0, dtype=dtype, device="cuda")
        evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=dx, act=evox_gpu.ACT_TANH,
                                  off=torch.tensor(off, dtype=torch.int32, device="cuda"))
        d = s["dy"].double() * nr.slope64(s["z"].double(), "tanh")
        for a, e, g in mine:
            if off[0] < 0 and g == 2:
                continue  # (rows of two networks)
            want = d[a:e] @ s["w"][g].double()
            close(dx[a:e], want, 1e-5 * (d[a:e].abs() @ s["w"][g].double().abs()), dtype, f"{off} {g}")
        assert off[0] < 0 or ((dx[:2] == 7).all() and (dx[35:] == 7).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_rows_with_infinities(evox_gpu, dtype):
    s = layer(dtype, [20, 25], 200, 260, seed=121)
    s["dy"][3, 5], s["dy"][7, 6], s["dy"][29, 8] = float("inf"), float("nan"), -float("inf")
    dx = filled(45, 200, dtype)
    evox_gpu.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=dx, off=s["off"], act=evox_gpu.ACT_SILU)
    d = s["dy"].double() * nr.slope64(s["z"].double(), "silu")
    for g, (a, e) in enumerate(s["spans"]):
        got, want = dx[a:e].double(), d[a:e] @ s["w"][g].double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        inf = torch.isinf(want)
        assert torch.equal(got[inf], want[inf]) and inf.any()
