"""The layers, norms and losses of a population of networks in 64 bits on the
CPU, written from their definitions, and the inputs their tests use."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # unit roundoff, of 24, 8 and 11 bits
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = ["none", "relu", "tanh", "gelu", "silu"]
U32 = U[torch.float32]


def spans(counts=None, G=None, M=None):
    """[(first row, end)] per network."""
    if counts is None:
        counts = [M // G] * G
    out, a = [], 0
    for c in counts:
        out.append((a, a + c))
        a += c
    return out


def offsets(counts, device="cuda"):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32, device=device)


def act64(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "tanh":
        return torch.tanh(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z.clone()


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "tanh":
        return 1 / torch.cosh(z) ** 2
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def rows_view(rng, G, n, dtype, lead=0, scale=1.0, pad=3):
    """[G, n] parameters inside the rows of a wider matrix (odd places and pitch)."""
    P = torch.randn(G, lead + n + pad, generator=rng, dtype=torch.float32).mul_(scale).to(dtype).cuda()
    return P[:, lead:lead + n]


def acts_view(rng, M, n, dtype, pad=0, scale=1.0):
    return torch.randn(M, n + pad, generator=rng, dtype=torch.float32).mul_(scale).to(dtype).cuda()[:, :n]


def linear64(x, w, b, spans_, shared):
    """z and the sum of the magnitudes of its terms."""
    x, w, b = x.double().cpu(), w.double().cpu(), None if b is None else b.double().cpu()
    M = spans_[-1][1]
    z, mag = torch.zeros(M, w.shape[1], dtype=torch.float64), torch.zeros(M, w.shape[1], dtype=torch.float64)
    for g, (a, e) in enumerate(spans_):
        xg = x if shared else x[a:e]
        z[a:e], mag[a:e] = xg @ w[g].t(), xg.abs() @ w[g].abs().t()
        if b is not None:
            z[a:e] += b[g]
            mag[a:e] += b[g].abs()
    return z, mag


def sum_bound(K, mag):
    """Of a sum of K products in fp32 in any order, each product from operands
    split into pieces that keep 22 bits of it at least."""
    return (K + 2) * U32 / (1 - (K + 2) * U32) * mag + 2.0 ** -22 * mag


def assert_close(got, want, bound, dtype, what):
    """|got - want| <= bound + one rounding to the element type."""
    got = got.double().cpu()
    limit = bound + (want.abs() + bound) * U[dtype] * 1.0001 + TINY[dtype]
    bad = ~((got - want).abs() <= limit)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, e.g. {got[bad][:3].tolist()} for "
                           f"{want[bad][:3].tolist()} +- {limit[bad][:3].tolist()}")
