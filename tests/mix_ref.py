"""The gate, the sort and the moves of a mixture of networks and the optimizer's step in
64 bits on the CPU, written from their definitions."""
import math

import torch


def order_key(z):
    """Logits as the gate orders them: NaN above +inf, -0 as 0."""
    z = z.double() + 0.0
    return torch.where(z.isnan(), torch.full_like(z, math.inf), z), z.isnan()


def gate64(z, k, over):
    """ids and weights of the k largest of every row, slot by slot."""
    T, G = z.shape
    key, nan = order_key(z.cpu())
    ids = torch.full((T, k), -1, dtype=torch.int32)
    for t in range(T):
        # Python's sort is stable: equal logits stay in the columns' order
        order = sorted((c for c in range(G) if key[t, c] > -math.inf), key=lambda c: (not nan[t, c], -float(key[t, c])))
        for j, c in enumerate(order[:k]):
            ids[t, j] = c
    return ids, gate_weights64(z, ids, over)


def gate_weights64(z, ids, over):
    z, ids = z.cpu().double(), ids.cpu().long()
    there = ids >= 0
    chosen = torch.where(there, z.gather(1, ids.clamp_min(0)), torch.full((), -math.inf, dtype=torch.float64))
    bad = (z.isnan() | (z == math.inf)).any(1, keepdim=True)
    # (not by the sum's logarithm: beside a logit of 1e38 it is lost, and four equal ones
    # would have weight 1 each)
    top = z.max(1, keepdim=True).values
    top = torch.where(top.isfinite(), top, torch.zeros_like(top))
    e = torch.exp(chosen - top)
    total = (e if over == "chosen" else torch.exp(z - top)).sum(1, keepdim=True)
    w = torch.where(there, e / total, torch.zeros_like(chosen))
    return torch.where(bad & there, torch.full_like(w, math.nan), w)


def gate_grad64(z, ids, w, dw, over):
    """dz, S's magnitude sum and the softmax over the row."""
    z, ids, w, dw = z.cpu().double(), ids.cpu().long(), w.cpu().double(), dw.cpu().double()
    T, G = z.shape
    there = (ids >= 0) & (ids < G)
    wd = torch.where(there, w * dw, torch.zeros_like(w))
    S, mag = wd.sum(1, keepdim=True), wd.abs().sum(1, keepdim=True)
    p = torch.zeros_like(z)
    if over == "all":
        p = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
    dz = -p * S
    for j in range(ids.shape[1]):
        at = ids[:, j].clamp(0, G - 1)
        rows = there[:, j]
        dz[rows, at[rows]] = (w[:, j:j + 1] * (dw[:, j:j + 1] - S))[rows, 0]
    return dz, S, mag, p


def route64(ids, G):
    """off, pos and the sorted slots."""
    flat = ids.cpu().flatten().tolist()
    rows = [[] for _ in range(G)]
    for slot, g in enumerate(flat):
        if 0 <= g < G:
            rows[g].append(slot)
    off, src = [0], []
    for r in rows:
        src += r
        off.append(len(src))
    pos = [-1] * len(flat)
    for m, slot in enumerate(src):
        pos[slot] = m
    return torch.tensor(off, dtype=torch.int32), torch.tensor(pos, dtype=torch.int32).view(ids.shape), src


def adamw64(p, g, m, v, t, lr, b1, b2, eps, decay):
    """p, m, v after step t, and the magnitudes of m's terms."""
    p, g, m, v = (x.double().cpu() for x in (p, g, m, v))
    mag = (b1 * m).abs() + ((1 - b1) * g).abs()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    den = torch.sqrt(v / (1 - b2 ** t)) + eps
    return p - lr * decay * p - lr * m / (1 - b1 ** t) / den, m, v, mag, lr / (1 - b1 ** t) / den
