"""A mixture of the population's networks and the step that trains it, as a program calls them.

Every row of the data goes to the k networks that a gate chooses for it; the
rows are brought into the networks' grouping (where their layers run) and
back; an optimizer updates parameters from their gradients.  The operators are

  gate          the k largest logits of a row and their softmax weights
  gate_grad     the logits' gradient from the weights'
  dispatch      slots (row, choice) sorted by network, rows moved to their places
  combine       y_t = sum_j w_tj xs[pos_tj] + r_t
  combine_grad  dxs[pos_tj] = w_tj dy_t, dw_tj = <dy_t, xs[pos_tj]>
  adamw         one step over many tensors, states in 32 or in 8 bits

listed() holds the sizes that are timed, draw() takes further ones from the
same ranges, run() makes one call (or, where `own` is false, computes the same
with elementary torch operations in 32 bits), exact() computes it in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK, TOP = 256, 448.0  # elements per scale of an 8-bit state; the largest e4m3 number


def _rows(op, dtype, T, G, k, D=0, over="chosen", drop=0.0, weights=True, residual=False, pad=0, name=None):
    c = {"op": op, "dtype": dtype, "T": T, "G": G, "k": k, "D": D, "over": over, "drop": drop, "weights": weights,
         "residual": residual, "pad": pad}
    return c if name is None else dict(c, name=name)


def _adamw(dtype, bits, kind, count, n, master=False, lead=0, name=None):
    c = {"op": "adamw", "dtype": dtype, "bits": bits, "kind": kind, "count": count, "n": n, "master": master,
         "lead": lead}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one observation, two of 64 networks: all latency
        _rows("gate", "f32", 1, 64, 2, name="gate_f32_1x64_k2"),
        # a training batch's gate, weights over all networks
        _rows("gate", "bf16", 65_536, 256, 8, over="all", name="gate_bf16_65536x256_k8"),
        # its gradient over a large population, an odd one, half precision
        _rows("gate_grad", "f16", 20_000, 1001, 4, over="all", name="gate_grad_f16_20000x1001_k4"),
        # one row to eight of 256 networks: all latency
        _rows("dispatch", "bf16", 1, 256, 8, 2048, weights=False, name="dispatch_bf16_1x2048_k8"),
        # odd rows, some of which a gate with a mask gave fewer networks
        _rows("dispatch", "f32", 10_007, 100, 2, 1001, drop=0.05, weights=False, name="dispatch_f32_10007x1001_k2"),
        # the largest: a batch to eight networks each
        _rows("dispatch", "bf16", 32_768, 64, 8, 2048, weights=False, name="dispatch_bf16_32768x2048_k8"),
        # back from the networks, added to a residual, odd sizes
        _rows("combine", "f32", 10_007, 100, 2, 1001, drop=0.05, residual=True, name="combine_f32_10007x1001_k2"),
        # the largest batch back
        _rows("combine", "bf16", 32_768, 64, 8, 2048, name="combine_bf16_32768x2048_k8"),
        # the gradient towards the networks' rows and the weights, half precision
        _rows("combine_grad", "f16", 16_384, 64, 4, 4096, name="combine_grad_f16_16384x4096_k4"),
        # 4096 policies of 1,830 parameters: one step of the population's rows
        _adamw("f32", 32, "rows", 4096, 1830, lead=26, name="adamw_f32_rows_4096x1830"),
        # 32 small layers in 16 bits with their 32-bit copies: 128 tensors, latency
        _adamw("bf16", 32, "layers", 32, 32, master=True, name="adamw_bf16_master_32_layers_32"),
        # 24 large layers in 16 bits, states in 8: 96 tensors, 100 million parameters
        _adamw("bf16", 8, "layers", 24, 2048, name="adamw_bf16_8bit_24_layers_2048"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST, MOST_GATE = 1.2e9, 1.5e8  # bytes


def draw(rng):
    op = rng.choice(["gate", "dispatch", "combine", "adamw"] * 2 + ["gate_grad", "combine_grad"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    while True:
        if op == "adamw":
            bits, master = rng.choice([32, 8]), dtype != "f32" and rng.random() < 0.5
            if rng.random() < 0.5:
                c = _adamw(dtype, bits, "rows", _log(rng, 1, 16_384), _log(rng, 1, 32_768), master, rng.randrange(100))
            else:
                c = _adamw(dtype, bits, "layers", _log(rng, 1, 64), _log(rng, 1, 4096), master)
        elif op.startswith("gate"):
            # (of one network, and of one choice that is the whole softmax, nothing depends on the inputs)
            G, over = _log(rng, 2, 16_384), rng.choice(["chosen", "all"])
            c = _rows(op, dtype, _log(rng, 1, 131_072), G, min(G, _log(rng, 2 if over == "chosen" else 1, 32)), 0, over,
                      pad=rng.choice([0, rng.randrange(40)]))
        else:
            T, G = _log(rng, 1, 131_072), _log(rng, 1, 16_384)
            c = _rows(op, dtype, T, G, min(G, _log(rng, 1, 16)), _log(rng, 1, 8192),
                      drop=rng.choice([0.0, 0.05, 0.5] if T >= 16 else [0.0]),
                      weights=rng.random() < (0.2 if op == "dispatch" else 0.8),
                      residual=op == "combine" and rng.random() < 0.4, pad=rng.choice([0, rng.randrange(40)]))
        if work(c)["bytes"] <= (MOST_GATE if op.startswith("gate") else MOST):
            return c


def _sizes(case):
    """Elements of the tensors of a step, each as (rows, length of a row)."""
    if case["kind"] == "rows":
        return [(case["count"], case["n"])]
    n = case["n"]
    return [(1, n * n), (1, n), (1, n), (1, n)] * case["count"]


def work(case):
    """Each input read once and each output written once."""
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op == "adamw":
        sizes = _sizes(case)
        N, blocks = sum(r * n for r, n in sizes), sum(r * -(-n // BLOCK) for r, n in sizes)
        own_bytes = e + 8 if case["master"] else 2 * e
        state = 16 * N if case["bits"] == 32 else 4 * N + 16 * blocks
        return {"bytes": N * (own_bytes + e) + state, "flops": 15.0 * N}
    T, G, k, D = case["T"], case["G"], case["k"], case["D"]
    n = T * k
    kept = n * (1 - case["drop"])
    if op == "gate":
        return {"bytes": e * T * G + 8 * n, "flops": 5.0 * T * G}
    if op == "gate_grad":
        return {"bytes": e * T * G * (2 if case["over"] == "all" else 1) + 12 * n, "flops": 6.0 * T * G}
    w = 4 * n if case["weights"] else 0
    if op == "dispatch":
        return {"bytes": 12 * n + 4 * (G + 1) + w + e * D * (T + kept), "flops": kept * D if w else 0.0}
    if op == "combine":
        return {"bytes": 4 * n + w + e * D * (T * (2 if case["residual"] else 1) + kept), "flops": 2.0 * kept * D}
    return {"bytes": 8 * n + w + e * D * (T + 2 * kept), "flops": 3.0 * kept * D}


def _choices(case, g):
    """ids [T, k]: k different networks per row, some networks far more often
    than others; a share of the slots without one."""
    T, G, k = case["T"], case["G"], case["k"]
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
    first = (u * u * G).long().clamp_(max=G - 1)
    step = torch.randint(1, max(1, (G - 1) // k) + 1, (T,), generator=g, device=DEV)
    ids = (first[:, None] + step[:, None] * torch.arange(k, device=DEV)) % G
    gone = torch.rand(T, k, generator=g, device=DEV) < case["drop"]
    return torch.where(gone, torch.full_like(ids, -1), ids).int()


def _places(ids, G):
    """off, pos and src of slots sorted by network, within one in their order."""
    flat = ids.flatten().long()
    key = torch.where((flat >= 0) & (flat < G), flat, torch.full_like(flat, G))
    key, order = torch.sort(key, stable=True)
    off = torch.searchsorted(key, torch.arange(G + 1, device=DEV))
    kept = key < G
    at = torch.arange(flat.numel(), device=DEV)
    pos = torch.empty_like(flat)
    pos[order] = torch.where(kept, at, torch.full_like(at, -1))
    return off.int(), pos.int().view(ids.shape), torch.where(kept, order, torch.zeros_like(order)).int()


def prepare(case, seed):
    """Inputs as the path meets them: logits and rows of unit scale, weights
    that are a softmax, gradients and optimizer states in mid-training; and the
    output buffers and handles that a program keeps."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dt, op = DTYPES[case["dtype"]], case["op"]
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32)
    s = {"case": case}
    if op == "adamw":
        return _prepare_adamw(s, g, dt, normal)
    T, G, k, D, pad = case["T"], case["G"], case["k"], case["D"], case["pad"]
    rows = lambda M, n: normal(M, n + pad).to(dt)[:, :n]
    softmax = lambda: torch.softmax(normal(T, k), 1)
    new = lambda *shape, d=dt: torch.zeros(*shape, device=DEV, dtype=d)
    if op.startswith("gate"):
        s["z"] = rows(T, G)
        # a mask leaves some networks out of some rows, and nothing of a few
        s["z"].masked_fill_(torch.rand(T, G, generator=g, device=DEV) < 0.02, -math.inf)
        s["z"][torch.rand(T, generator=g, device=DEV) < 0.001] = -math.inf
        if op == "gate":
            s["ids"], s["w"] = new(T, k, d=torch.int32), new(T, k, d=torch.float32)
        else:
            s["ids"], s["w"] = _top(s["z"].float(), k, case["over"])
            s["dw"], s["dz"] = normal(T, k), new(T, G)
        return s
    ids = _choices(case, g)
    s["w"] = softmax() if case["weights"] else None
    if op == "dispatch":
        s["ids"], s["x"], s["xs"] = ids, rows(T, D), new(T * k, D)
        s["off"], s["pos"], s["src"] = new(G + 1, d=torch.int32), new(T, k, d=torch.int32), new(T * k, d=torch.int32)
        if own:
            import paper_2301_12457_amd as evox
            s["scratch"] = evox.evox_route_scratch(s["ids"], s["off"])
        return s
    s["pos"] = _places(ids, G)[1]
    s["xs"] = rows(T * k, D)
    if op == "combine":
        s["r"], s["y"] = rows(T, D) if case["residual"] else None, new(T, D)
    else:
        s["dy"], s["dxs"], s["dw"] = rows(T, D), new(T * k, D), new(T, k, d=torch.float32)
    return s


def _prepare_adamw(s, g, dt, normal):
    case = s["case"]
    sizes = _sizes(case)
    N = sum(r * n for r, n in sizes)
    if case["kind"] == "rows":
        (G, n), pitch = sizes[0], (case["lead"] + case["n"] + 31) // 32 * 32
        s["p"], s["g"] = normal(G, pitch).to(dt), normal(G, pitch).mul_(0.02).to(dt)
        s["params"], s["grads"] = ([t[:, case["lead"]:case["lead"] + n]] for t in (s["p"], s["g"]))
    else:
        s["p"], s["g"] = normal(N).to(dt), normal(N).mul_(0.02).to(dt)
        cut = lambda t: [v.view(r, n) for v, (r, n) in zip(t.split([r * n for r, n in sizes]), sizes)]
        s["params"], s["grads"] = cut(s["p"]), cut(s["g"])
    m, v = normal(N).mul_(0.006), normal(N).mul_(0.02).square_().mul_(torch.rand(N, generator=g, device=DEV))
    st = {"t": torch.tensor([1000], device=DEV)}
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
    else:
        st["m"], st["m_scale"] = _to8(m, sizes, False)
        st["v"], st["v_scale"] = _to8(v.sqrt_(), sizes, True)
    if case["master"]:
        flat = torch.cat([p.float().flatten() for p in s["params"]])
        st["master"] = flat * (1 + 0.001 * torch.rand(N, generator=g, device=DEV))
    if own:
        import paper_2301_12457_amd as evox
        s["opt"] = evox.AdamW(s["params"], s["grads"], lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                              bits=case["bits"], master=case["master"])
        for name, t in st.items():
            s["opt"].state[name].copy_(t)
        st = s["opt"].state
    s["state"] = st
    return s


def _results(s):
    """Parameters and states after a step (8-bit ones as e4m3 numbers and their
    scales, whose products they stand for)."""
    return dict({name: t for name, t in s["state"].items() if name != "t"}, p=s["p"])


def _call(s):
    import paper_2301_12457_amd as evox
    case = s["case"]
    op = case["op"]
    if op.startswith("gate"):
        over = evox.GATE_ALL if case["over"] == "all" else evox.GATE_CHOSEN
    if op == "gate":
        evox.evox_gate(s["z"], s["ids"], s["w"], over=over)
        return {"ids": s["ids"], "w": s["w"]}
    if op == "gate_grad":
        evox.evox_gate_grad(s["z"], s["ids"], s["w"], s["dw"], s["dz"], over=over)
        return {"dz": s["dz"]}
    if op == "dispatch":
        evox.evox_route(s["ids"], s["off"], s["pos"], src=s["src"], scratch=s["scratch"])
        evox.evox_dispatch(s["x"], s["pos"], s["xs"], w=s["w"])
        return {"off": s["off"], "pos": s["pos"], "src": s["src"], "xs": s["xs"]}
    if op == "combine":
        evox.evox_combine(s["xs"], s["pos"], s["y"], w=s["w"], r=s["r"])
        return {"y": s["y"]}
    if op == "combine_grad":
        evox.evox_combine_grad(s["xs"], s["pos"], s["dy"], w=s["w"], dxs=s["dxs"], dw=s["dw"])
        return {"dxs": s["dxs"], "dw": s["dw"]}
    s["opt"].step()
    return _results(s)


# ---------------------------------------------------------------------------
# The plain form: elementary torch operations in 32 bits, rounded at the end.
# ---------------------------------------------------------------------------
def _top(z, k, over):
    """The k largest of every row, ties to the lower index, and their weights."""
    top, ids = torch.sort(z, dim=1, descending=True, stable=True)
    first, top, ids = top[:, :1], top[:, :k], ids[:, :k]
    there = top > -math.inf
    first = torch.where(first > -math.inf, first, torch.zeros_like(first))
    e = torch.exp(top - first)
    total = (torch.exp(z - first) if over == "all" else e).sum(1, keepdim=True)
    w = torch.where(there, e / total, torch.zeros_like(e))
    return torch.where(there, ids, torch.full_like(ids, -1)).int(), w


def _to8(x, sizes, root):
    """e4m3 numbers and a scale for each 256 elements of a row, its largest
    magnitude over 448.  root: roots of second moments, above 0 never to 0."""
    b = _blocks(x, sizes)
    most = b.abs().amax(1, keepdim=True)
    q = (b * torch.where(most > 2.0 ** -100, TOP / most, torch.zeros_like(most))).to(torch.float8_e4m3fn)
    if root:
        code = q.view(torch.uint8)
        q = torch.where((b > 0) & (code == 0), torch.ones_like(code), code).view(torch.float8_e4m3fn)
    return _unblock(q.view(torch.uint8), sizes).view(torch.float8_e4m3fn), (most * (1 / TOP))[:, 0]


def _from8(q, scale, sizes):
    return _unblock(_blocks(q.float(), sizes) * scale[:, None], sizes)


def _blocks(x, sizes):
    """[blocks, 256], a row's last block filled with 0."""
    if all(n % BLOCK == 0 for _, n in sizes):
        return x.view(-1, BLOCK)
    fill = lambda t, n: torch.nn.functional.pad(t, (0, -n % BLOCK)).view(-1, BLOCK)
    return torch.cat([fill(t.view(r, n), n) for t, (r, n) in zip(x.split([r * n for r, n in sizes]), sizes)])


def _unblock(b, sizes):
    if all(n % BLOCK == 0 for _, n in sizes):
        return b.reshape(-1)
    per = [r * -(-n // BLOCK) for r, n in sizes]
    return torch.cat([t.view(r, -1)[:, :n].flatten() for t, (r, n) in zip(b.split(per), sizes)])


def _plain_adamw(s):
    case, st = s["case"], s["state"]
    sizes = _sizes(case)
    st["t"] += 1
    t = st["t"].double()
    rate, root = (LR / (1 - BETA1 ** t)).float(), (1 / torch.sqrt(1 - BETA2 ** t)).float()
    # all tensors of a step as one vector (they lie one behind the other; a population's rows have gaps)
    flat = (lambda t: t) if case["kind"] == "layers" else lambda t: t[:, case["lead"]:case["lead"] + case["n"]].reshape(-1)
    g = flat(s["g"]).float()
    m, v = st["m"], st["v"]
    if case["bits"] == 8:
        m, v = _from8(m, st["m_scale"], sizes), _from8(v, st["v_scale"], sizes).square()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    r = torch.sqrt(v)
    p = st["master"] if case["master"] else flat(s["p"]).float()
    p = (p - p * (LR * DECAY)) - rate * (m / (r * root + EPS))
    if case["bits"] == 8:
        (m, ms), (v, vs) = _to8(m, sizes, False), _to8(r, sizes, True)
        st["m_scale"].copy_(ms)
        st["v_scale"].copy_(vs)
    st["m"].copy_(m)
    st["v"].copy_(v)
    if case["master"]:
        st["master"].copy_(p)
    if case["kind"] == "rows":
        s["params"][0].copy_(p.view(case["count"], case["n"]))
    else:
        s["p"].copy_(p)
    return _results(s)


def _plain(s):
    case = s["case"]
    op, dt, G, k = case["op"], DTYPES[case["dtype"]], case.get("G"), case.get("k")
    if op == "adamw":
        return _plain_adamw(s)
    if op == "gate":
        ids, w = _top(s["z"].float(), k, case["over"])
        return {"ids": ids, "w": w}
    if op == "gate_grad":
        z, ids, w, dw = s["z"].float(), s["ids"], s["w"], s["dw"]
        there = ids >= 0
        at = torch.where(there, ids, torch.zeros_like(ids)).long()
        S = (w * dw).sum(1, keepdim=True)
        part = torch.where(there, w * dw, torch.zeros_like(w))
        if case["over"] == "all":
            top = z.max(1, keepdim=True).values
            e = torch.exp(z - torch.where(top > -math.inf, top, torch.zeros_like(top)))
            total = e.sum(1, keepdim=True)
            dz = -S * (e / torch.where(total > 0, total, torch.ones_like(total)))
        else:
            part = part - w * S
            dz = torch.zeros_like(z)
        return {"dz": dz.scatter_add_(1, at, part).to(dt)}
    if op == "dispatch":
        off, pos, src = _places(s["ids"], G)
        there = pos >= 0
        x = s["x"].float()[:, None, :].expand(-1, k, -1)[there]
        if s["w"] is not None:
            x = x * s["w"][there][:, None]
        xs = torch.zeros(pos.numel(), x.shape[1], dtype=dt, device=DEV)
        xs[pos[there].long()] = x.to(dt)
        return {"off": off, "pos": pos, "src": src, "xs": xs}
    pos = s["pos"].long()
    there = (pos >= 0)[:, :, None]
    rows = s["xs"].float()[pos.clamp_min(0)]
    rows = torch.where(there, rows, torch.zeros_like(rows))
    if op == "combine":
        if s["w"] is not None:
            rows = rows * s["w"][:, :, None]
        y = rows.sum(1)
        return {"y": (y if s["r"] is None else y + s["r"].float()).to(dt)}
    dy = s["dy"].float()[:, None, :]
    dw = (rows * dy).sum(2)
    d = dy * (there.float() if s["w"] is None else s["w"][:, :, None])
    dxs = torch.zeros(s["xs"].shape, dtype=dt, device=DEV)
    dxs[pos[there[:, :, 0]]] = d.expand(-1, k, -1)[there[:, :, 0]].to(dt)
    return {"dxs": dxs, "dw": dw}


def run(state):
    return _call(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# In 64 bits, from the definitions: a choice at a time, rows in pieces, tensors
# one by one.
# ---------------------------------------------------------------------------
def _pieces(total, width):
    step = max(1, int(5e7 // max(1, width)))
    return [slice(a, min(total, a + step)) for a in range(0, total, step)]


def _exact_gate(case, s):
    T, G, k = case["T"], case["G"], case["k"]
    w = torch.zeros(T, k, dtype=torch.float64, device=DEV)
    for sl in _pieces(T, G):
        z = s["z"][sl].double()
        left = z.clone()
        total = torch.zeros(len(z), dtype=torch.float64, device=DEV)
        top = z.max(1).values
        base = torch.where(top.isinf(), torch.zeros_like(top), top)
        for j in range(k):
            value, at = left.max(1)
            left.scatter_(1, at[:, None], -math.inf)
            w[sl, j] = torch.exp(value - base)
            total += w[sl, j]
        if case["over"] == "all":
            total = torch.exp(z - base[:, None]).sum(1)
        w[sl] /= torch.where(total > 0, total, torch.ones_like(total))[:, None]
    return {"ids": None, "w": w}


def _exact_gate_grad(case, s):
    T, G = case["T"], case["G"]
    dz = torch.zeros(T, G, dtype=torch.float64, device=DEV)
    for sl in _pieces(T, G):
        z, ids, dw = s["z"][sl].double(), s["ids"][sl].long(), s["dw"][sl].double()
        chosen = torch.zeros(len(z), G + 1, dtype=torch.float64, device=DEV)  # (the last column: no choice)
        slope = torch.zeros_like(chosen)
        at = torch.where(ids >= 0, ids, torch.full_like(ids, G))
        chosen.scatter_(1, at, 1.0)
        slope.scatter_(1, at, dw)
        chosen, slope = chosen[:, :G], slope[:, :G]
        if case["over"] == "chosen":
            z = torch.where(chosen > 0, z, torch.full_like(z, -math.inf))
        p = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)  # (rows that a mask leaves nothing of)
        dz[sl] = p * (slope - (p * slope * chosen).sum(1, keepdim=True))
    return {"dz": dz}


def _exact_dispatch(case, s):
    T, G, k, D = case["T"], case["G"], case["k"], case["D"]
    slot = torch.arange(T * k, device=DEV)
    ids = s["ids"].flatten().long()
    slot = slot[(ids >= 0) & (ids < G)]
    slot = slot[torch.argsort(ids[slot] * (T * k) + slot)]
    xs = torch.zeros(T * k, D, dtype=torch.float64, device=DEV)
    for sl in _pieces(len(slot), D):
        row = s["x"][torch.div(slot[sl], k, rounding_mode="floor")].double()
        xs[sl] = row if s["w"] is None else row * s["w"].flatten()[slot[sl]].double()[:, None]
    return {"off": None, "pos": None, "src": None, "xs": xs}


def _exact_combine(case, s):
    T, k, D = case["T"], case["k"], case["D"]
    forward = case["op"] == "combine"
    y = torch.zeros(T if forward else T * k, D, dtype=torch.float64, device=DEV)
    dw = torch.zeros(T, k, dtype=torch.float64, device=DEV)
    for sl in _pieces(T, D):
        if forward and s["r"] is not None:
            y[sl] = s["r"][sl].double()
        for j in range(k):
            at = s["pos"][sl, j].long()
            t = torch.arange(T, device=DEV)[sl][at >= 0]
            at = at[at >= 0]
            w = s["w"][t, j].double()[:, None] if s["w"] is not None else 1.0
            if forward:
                y[t] += w * s["xs"][at].double()
            else:
                dy = s["dy"][t].double()
                y[at] = w * dy
                dw[t, j] = torch.linalg.vecdot(dy, s["xs"][at].double())
    return {"y": y} if forward else {"dxs": y, "dw": dw}


def _exact_adamw(case, s):
    st = s["state"]
    t = int(st["t"]) + 1
    out = {name: torch.zeros(x.shape, dtype=torch.float64, device=DEV) for name, x in st.items() if name != "t"}
    out["p"] = s["p"].double()
    at, block = 0, 0
    for i, (r, n) in enumerate(_sizes(case)):
        N, per = r * n, -(-n // BLOCK)
        nb = r * per
        mine, blocks = slice(at, at + N), slice(block, block + nb)
        spread = lambda x: x[blocks].double().view(r, per).repeat_interleave(BLOCK, 1)[:, :n]
        m, v = st["m"][mine].double().view(r, n), st["v"][mine].double().view(r, n)
        if case["bits"] == 8:
            m, v = m * spread(st["m_scale"]), (v * spread(st["v_scale"])) ** 2
        g = s["grads"][i].double()
        p = st["master"][mine].view(r, n).double() if case["master"] else s["params"][i].double()
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g.pow(2)
        p = p * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
        for name, x in (("m", m), ("v", v)):
            if case["bits"] == 8:
                x = x if name == "m" else x.sqrt()
                filled = torch.zeros(r, per * BLOCK, dtype=torch.float64, device=DEV)
                filled[:, :n] = x
                most = filled.view(r, per, BLOCK).abs().max(2).values
                out[name + "_scale"][blocks] = most.flatten() / TOP
                ratio = torch.where(most > 0, TOP / most, most).repeat_interleave(BLOCK, 1)[:, :n]
                # to three bits behind the leading one, 2^-9 at the least
                q = x * ratio
                unit = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
                q = torch.round(q / unit) * unit
                x = torch.where((x > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q) if name == "v" else q
            out[name][mine] = x.flatten()
        if case["master"]:
            out["master"][mine] = p.flatten()
        if case["kind"] == "rows":
            out["p"][:, case["lead"]:case["lead"] + n] = p
        else:
            out["p"][mine] = p.flatten()
        at, block = at + N, block + nb
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "gate":
        return _exact_gate(case, s)
    if op == "gate_grad":
        return _exact_gate_grad(case, s)
    if op == "dispatch":
        return _exact_dispatch(case, s)
    return _exact_adamw(case, s) if op == "adamw" else _exact_combine(case, s)
