"""The layers of a population of networks, as a program that evolves or trains one calls them.

A population X[G, ldp] holds one network per row; the parameters of a layer
lie at a fixed offset of every row.  Network g owns the rows off[g] .. off[g+1)
of the activations.  The operators are

  linear          z = x W_g^T + b_g, y = act(z) + r
  linear_grad     d = dy act'(z): dx = d W_g, dW_g = d^T x, db_g = sum of d
  layernorm       y = (x - mean) / sqrt(var + eps) gamma_g + beta_g
  layernorm_grad  dx, dgamma_g, dbeta_g
  xent            fit_g = mean cross-entropy of a network's rows, and its gradient

listed() holds the sizes that are timed, draw() takes further ones from the
same ranges, run() makes one call (or, where `own` is false, computes the same
with elementary torch operations in 32 bits), exact() computes it in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ("none", "relu", "tanh", "gelu", "silu")
EPS = 1e-5


def _case(op, dtype, G, M, n_in, n_out=0, act="none", ragged=False, residual=False, shared=False, save=False,
          lead=0, name=None):
    c = {"op": op, "dtype": dtype, "G": G, "M": M, "n_in": n_in, "n_out": n_out, "act": act, "ragged": ragged,
         "residual": residual, "shared": shared, "save": save, "lead": lead}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one control step of 4096 policies of 1,830 parameters (17-32-32-6):
        # the middle layer, one observation each, weights read from the rows of
        # the population; all latency
        _case("linear", "f32", 4096, 4096, 32, 32, "tanh", lead=576, name="linear_f32_step_4096x1_32x32"),
        # a generation of 100 wide networks whose episodes ended at different
        # times: ragged rows, an odd fan-in, a residual
        _case("linear", "f32", 100, 10_000, 1001, 1000, "relu", ragged=True, residual=True,
              name="linear_f32_ragged_100x100_1001x1000"),
        # every individual on the same batch of 100 observations, kept for the
        # backward pass
        _case("linear", "f16", 1000, 100_000, 100, 100, "silu", shared=True, save=True,
              name="linear_f16_shared_1000x100_100x100"),
        # single rows through 256 large networks: as fast as the weights arrive
        _case("linear", "bf16", 256, 256, 2048, 2048, "gelu", name="linear_bf16_step_256x1_2048x2048"),
        # few large networks in 32 bits
        _case("linear", "f32", 16, 4096, 2048, 2048, "none", name="linear_f32_16x256_2048x2048"),
        # the largest: 16 networks, ragged, two thousand rows each
        _case("linear", "bf16", 16, 32_768, 4096, 4096, "gelu", ragged=True, residual=True,
              name="linear_bf16_ragged_16x2048_4096x4096"),
        # gradient of the 1,830-parameter policies' middle layer on 32 rows each
        _case("linear_grad", "f32", 4096, 131_072, 32, 32, "tanh", lead=576, name="linear_grad_f32_4096x32_32x32"),
        # gradient of a layer of 64 networks with ragged shares of the data
        _case("linear_grad", "bf16", 64, 32_768, 1024, 1024, "gelu", ragged=True,
              name="linear_grad_bf16_ragged_64x512_1024x1024"),
        # the norm before such layers, half precision
        _case("layernorm", "f16", 64, 65_536, 1024, name="layernorm_f16_64x1024_1024"),
        # its gradient, 32 bits, ragged and odd
        _case("layernorm_grad", "f32", 100, 20_000, 1001, ragged=True, name="layernorm_grad_f32_ragged_100x200_1001"),
        # fitness of 4096 small classifiers, ten classes, 32 samples each
        _case("xent", "f32", 4096, 131_072, 10, shared=True, name="xent_f32_shared_4096x32_10"),
        # fitness and gradient over the largest class count
        _case("xent", "bf16", 16, 8192, 32_768, ragged=True, name="xent_bf16_ragged_16x512_32768"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = {"bytes": 2.5e9, "flops": 1.1e12}


def draw(rng):
    op = rng.choice(["linear"] * 4 + ["linear_grad"] * 3 + ["layernorm", "layernorm_grad"] * 2 + ["xent"] * 2)
    dtype = rng.choice(["f32", "bf16", "f16"])
    act = rng.choice(ACTS) if op.startswith("linear") else "none"
    ragged = rng.random() < 0.5
    shared = not ragged and op in ("linear", "linear_grad", "xent") and rng.random() < 0.3
    residual, save = rng.random() < 0.4, rng.random() < 0.4
    lead = rng.choice([0, rng.randrange(1000)])
    G, rows = _log(rng, 1, 16_384), _log(rng, 1, 4096)
    if op.startswith("linear"):
        n_in, n_out = _log(rng, 1, 4096), _log(rng, 1, 4096)
    else:
        n_in, n_out = _log(rng, 2, 32_768), 0
    while True:
        M = G * rows
        if ragged and op != "xent":
            M = max(1, M - rng.randrange(1 + M // 7))
        c = _case(op, dtype, G, M, n_in, n_out, act, ragged, residual and op == "linear", shared,
                  save and op == "linear", lead)
        w = work(c)
        if w["bytes"] <= MOST["bytes"] and w["flops"] <= MOST["flops"] and M * max(n_in, n_out) <= 2.0e9:
            return c
        if G > 1 and rng.random() < 0.5:
            G = (G + 1) // 2
        elif rows > 1:
            rows = (rows + 1) // 2
        else:
            n_in = (n_in + 1) // 2
            n_out = (n_out + 1) // 2 if n_out else 0


def work(case):
    """Each input read once and each output written once; the products' operations."""
    e = 4 if case["dtype"] == "f32" else 2
    op, G, M, n_in, n_out = case["op"], case["G"], case["M"], case["n_in"], case["n_out"]
    xrows = M // G if case["shared"] else M
    if op == "linear":
        outs = M * n_out * (1 + case["save"] + case["residual"])
        return {"bytes": e * (xrows * n_in + G * (n_in + 1) * n_out + outs), "flops": 2.0 * M * n_in * n_out}
    if op == "linear_grad":
        z = 0 if case["act"] == "none" else M * n_out
        dx = 0 if case["shared"] else M * n_in
        w = 0 if case["shared"] else G * n_in * n_out
        return {"bytes": e * (xrows * n_in + w + z + M * n_out + dx + G * (n_in + 1) * n_out),
                "flops": (2.0 if case["shared"] else 4.0) * M * n_in * n_out}
    if op == "layernorm":
        return {"bytes": e * (2 * M * n_in + 2 * G * n_in) + 8 * M, "flops": 8.0 * M * n_in}
    if op == "layernorm_grad":
        return {"bytes": e * (3 * M * n_in + 3 * G * n_in) + 8 * M, "flops": 14.0 * M * n_in}
    return {"bytes": e * 2 * M * n_in + 4 * xrows + 4 * G, "flops": 8.0 * M * n_in}


def _offsets(case, g):
    """Rows of each network: between none and twice the mean, some none at all
    (for the loss every network has at least one row)."""
    G, M = case["G"], case["M"]
    u = torch.rand(G, generator=g, device=DEV, dtype=torch.float64)
    if case["op"] == "xent":
        inner = torch.floor(torch.cumsum(u, 0) / u.sum() * (M - G)).long() + torch.arange(1, G + 1, device=DEV)
    else:
        u = torch.where(u < 0.05, torch.zeros_like(u), u)
        inner = torch.floor(torch.cumsum(u, 0) / u.sum().clamp_min(1e-9) * M).long()
    off = torch.zeros(G + 1, dtype=torch.int32, device=DEV)
    off[1:] = inner.clamp(0, M).int()
    off[G] = M
    return off


def prepare(case, seed):
    """Inputs as the path meets them: activations of unit scale, weights scaled
    by the fan-in, 5 % of the labels out of range (unlabelled rows); and the
    output buffers and scratch that a program keeps."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    op, dt, G, M, n_in, n_out = (case["op"], DTYPES[case["dtype"]], case["G"], case["M"], case["n_in"],
                                 case["n_out"])
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32).to(dt)
    empty = lambda *s, d=dt: torch.empty(*s, device=DEV, dtype=d)
    s = {"case": case, "off": _offsets(case, g) if case["ragged"] else None}
    # the program that filled the offsets has the row counts on the host too
    s["bounds"] = s["off"].tolist() if case["ragged"] else [i * (M // G) for i in range(G + 1)]
    xrows = M // G if case["shared"] else M

    def rows_of(n):
        pitch = (case["lead"] + n + 31) // 32 * 32
        return normal(G, pitch)[:, case["lead"]:case["lead"] + n]

    if op in ("linear", "linear_grad"):
        s["x"] = normal(xrows, n_in)
        P = rows_of((n_in + 1) * n_out)
        s["w"] = P[:, :n_in * n_out].unflatten(1, (n_out, n_in))
        s["w"].mul_(n_in ** -0.5)
        s["b"] = P[:, n_in * n_out:]
        s["b"].mul_(0.1)
    if op == "linear":
        s["r"] = normal(M, n_out) if case["residual"] else None
        s["y"] = empty(M, n_out)
        s["z"] = empty(M, n_out) if case["save"] else None
    elif op == "linear_grad":
        s["z"] = normal(M, n_out) if case["act"] != "none" else None
        s["dy"] = normal(M, n_out)
        s["dx"] = None if case["shared"] else empty(M, n_in)
        s["dw"], s["db"] = empty(G, n_out, n_in), empty(G, n_out)
    elif op in ("layernorm", "layernorm_grad"):
        s["x"] = normal(M, n_in).mul_(1.5).add_(0.5)
        P = rows_of(2 * n_in)
        s["gamma"], s["beta"] = P[:, :n_in], P[:, n_in:]
        s["gamma"].mul_(0.2).add_(1.0)
        s["beta"].mul_(0.2)
        if op == "layernorm":
            s["y"] = empty(M, n_in)
            s["mean"], s["rstd"] = empty(M, d=torch.float32), empty(M, d=torch.float32)
        else:
            x32 = s["x"].float()
            s["mean"] = x32.mean(1)
            s["rstd"] = 1.0 / torch.sqrt((x32 - s["mean"][:, None]).square().mean(1) + EPS)
            s["dy"], s["dx"] = normal(M, n_in), empty(M, n_in)
            s["dgamma"], s["dbeta"] = empty(G, n_in), empty(G, n_in)
    else:
        s["logits"] = normal(M, n_in).mul_(2.0)
        lab = torch.randint(0, n_in, (xrows,), generator=g, device=DEV, dtype=torch.int32)
        drop = torch.rand(xrows, generator=g, device=DEV) < 0.05
        if case["ragged"]:
            drop[s["off"][:-1].long()] = False
        else:
            drop[::max(1, M // G)] = False
        s["labels"] = torch.where(drop, torch.full_like(lab, -1), lab)
        s["fit"], s["dz"] = empty(G, d=torch.float32), empty(M, n_in)
    if own:
        import paper_2301_12457_amd as evox
        s["scratch"] = None
        if op == "linear_grad":
            s["scratch"] = evox.evox_linear_grad_scratch(s["x"], s["w"], s["dy"])
        elif op == "layernorm_grad":
            s["scratch"] = evox.evox_layernorm_grad_scratch(s["x"], s["gamma"])
        elif op == "xent":
            s["scratch"] = evox.evox_xent_scratch(s["logits"], s["fit"])
    return s


def _call(s):
    import paper_2301_12457_amd as evox
    case = s["case"]
    op, act = case["op"], ACTS.index(case["act"])
    if op == "linear":
        evox.evox_linear(s["x"], s["w"], s["y"], b=s["b"], r=s["r"], z=s["z"], off=s["off"], act=act)
        return {"y": s["y"], "z": s["z"]} if case["save"] else {"y": s["y"]}
    if op == "linear_grad":
        evox.evox_linear_grad(s["x"], s["w"], s["dy"], z=s["z"], dx=s["dx"], dw=s["dw"], db=s["db"], off=s["off"],
                              act=act, scratch=s["scratch"])
        out = {"dw": s["dw"], "db": s["db"]}
        return out if case["shared"] else dict(out, dx=s["dx"])
    if op == "layernorm":
        evox.evox_layernorm(s["x"], s["gamma"], s["beta"], s["y"], mean=s["mean"], rstd=s["rstd"], off=s["off"],
                            eps=EPS)
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "layernorm_grad":
        evox.evox_layernorm_grad(s["x"], s["gamma"], s["mean"], s["rstd"], s["dy"], s["dx"], dgamma=s["dgamma"],
                                 dbeta=s["dbeta"], off=s["off"], scratch=s["scratch"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    evox.evox_xent(s["logits"], s["labels"], s["fit"], dz=s["dz"], off=s["off"], scratch=s["scratch"])
    return {"fit": s["fit"], "dz": s["dz"]}


# ---------------------------------------------------------------------------
# The plain form: elementary torch operations in 32 bits, rounded at the end.
# Few networks are a product each; many are one batched product, ragged rows
# padded to the longest.
# ---------------------------------------------------------------------------
LOOP = 64


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "tanh":
        return torch.tanh(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "tanh":
        return 1 - torch.tanh(z).square()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


class _Rows:
    """Rows of every network as a padded batch [G, n, .], and back."""

    def __init__(self, s):
        case = s["case"]
        self.G, self.M, self.even = case["G"], case["M"], not case["ragged"]
        if self.even:
            self.n = self.M // self.G
            return
        off = s["off"].long()
        self.n = max(1, max(b - a for a, b in zip(s["bounds"], s["bounds"][1:])))
        row = torch.arange(self.M, device=DEV)
        net = torch.searchsorted(off, row, right=True) - 1
        self.slot = net * self.n + row - off[net]

    def pad(self, t):
        if self.even:
            return t.reshape(self.G, self.n, -1)
        out = t.new_zeros(self.G * self.n, t.shape[1])
        out[self.slot] = t
        return out.view(self.G, self.n, -1)

    def flat(self, t):
        if self.even:
            return t.reshape(self.M, -1)
        return t.reshape(self.G * self.n, -1)[self.slot]


def _net_of_row(s):
    case = s["case"]
    row = torch.arange(case["M"], device=DEV)
    if not case["ragged"]:
        return row // (case["M"] // case["G"])
    return torch.searchsorted(s["off"].long(), row, right=True) - 1


def _sum_by_net(t, s):
    """[G, .] sums of the rows of each network, in 32 bits."""
    case = s["case"]
    if not case["ragged"]:
        return t.view(case["G"], case["M"] // case["G"], -1).sum(1)
    if case["G"] <= LOOP:
        return torch.stack([t[a:b].sum(0) for a, b in zip(s["bounds"], s["bounds"][1:])])
    return _Rows(s).pad(t).sum(1)


def _plain(s):
    case = s["case"]
    op, act, G, M = case["op"], case["act"], case["G"], case["M"]
    dt = DTYPES[case["dtype"]]
    spans = list(zip(s["bounds"], s["bounds"][1:]))
    if op == "linear":
        x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
        if G <= LOOP:
            z = torch.cat([(x if case["shared"] else x[a:e]) @ w[g].t() + b[g] for g, (a, e) in enumerate(spans)])
        elif case["shared"]:
            z = (torch.matmul(x, w.transpose(1, 2)) + b[:, None, :]).view(M, -1)
        else:
            R = _Rows(s)
            z = R.flat(torch.matmul(R.pad(x), w.transpose(1, 2)) + b[:, None, :])
        y = _act(z, act)
        if case["residual"]:
            y = y + s["r"].float()
        return {"y": y.to(dt), "z": z.to(dt)} if case["save"] else {"y": y.to(dt)}
    if op == "linear_grad":
        x, w, d = s["x"].float(), s["w"].float(), s["dy"].float()
        if act != "none":
            d = d * _slope(s["z"].float(), act)
        if G <= LOOP:
            dw = torch.stack([d[a:e].t() @ (x if case["shared"] else x[a:e]) for a, e in spans])
            dx = None if case["shared"] else torch.cat([d[a:e] @ w[g] for g, (a, e) in enumerate(spans)])
        else:
            R = _Rows(s)
            dp = R.pad(d)
            dw = torch.matmul(dp.transpose(1, 2), x if case["shared"] else R.pad(x))
            dx = None if case["shared"] else R.flat(torch.matmul(dp, w))
        out = {"dw": dw.to(dt), "db": _sum_by_net(d, s).to(dt)}
        return out if case["shared"] else dict(out, dx=dx.to(dt))
    if op == "layernorm":
        x, net = s["x"].float(), _net_of_row(s)
        mean = x.mean(1, keepdim=True)
        rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        y = (x - mean) * rstd * s["gamma"].float()[net] + s["beta"].float()[net]
        return {"y": y.to(dt), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "layernorm_grad":
        x, dy, net = s["x"].float(), s["dy"].float(), _net_of_row(s)
        rstd = s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        a = dy * s["gamma"].float()[net]
        dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
        return {"dx": dx.to(dt), "dgamma": _sum_by_net(dy * xh, s).to(dt), "dbeta": _sum_by_net(dy, s).to(dt)}
    z = s["logits"].float()
    lab = s["labels"].long()
    if case["shared"]:
        lab = lab.repeat(G)
    good = (lab >= 0) & (lab < case["n_in"])
    at = torch.where(good, lab, torch.zeros_like(lab))[:, None]
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    loss = (torch.log(total) + top - z.gather(1, at))[:, 0]
    count = _sum_by_net(good.float()[:, None], s)
    fit = _sum_by_net(torch.where(good, loss, torch.zeros_like(loss))[:, None], s) / count
    scale = good.float()[:, None] / count[_net_of_row(s)]
    dz = e / total
    dz.scatter_add_(1, at, torch.full_like(total, -1.0))
    return {"fit": fit[:, 0], "dz": (dz * scale).to(dt)}


def run(state):
    return _call(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# In 64 bits, network by network or in chunks of rows.
# ---------------------------------------------------------------------------
def _exact_act(z, act):
    """act(z) and its derivative."""
    one = torch.ones_like(z)
    if act == "relu":
        return torch.clamp_min(z, 0), torch.where(z > 0, one, 0 * one)
    if act == "tanh":
        e = torch.exp(-2 * z.abs())
        t = torch.sign(z) * (1 - e) / (1 + e)
        return t, 4 * e / (1 + e) ** 2
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) * (2 * math.pi) ** -0.5
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p + z * p * (1 - p)
    return z, one


def _blocks(s):
    """(networks, rows) a few at a time: the networks g0 .. g1 and, for even
    rows, all of their rows at once; else one network with rows at a time."""
    case = s["case"]
    G, M = case["G"], case["M"]
    if case["ragged"]:
        return [(g, g + 1, a, e) for g, (a, e) in enumerate(zip(s["bounds"], s["bounds"][1:])) if e > a]
    n = M // G
    size = max(case["n_in"] * max(1, case["n_out"]), n * max(case["n_in"], case["n_out"]))
    per = max(1, int(2e8 // size))
    return [(g, min(G, g + per), g * n, min(G, g + per) * n) for g in range(0, G, per)]


def exact(case, seed):
    s = prepare(case, seed)
    op, act, M, G = case["op"], case["act"], case["M"], case["G"]
    f64 = torch.float64
    new = lambda *shape: torch.empty(*shape, dtype=f64, device=DEV)
    if op == "linear":
        out = {"y": new(M, case["n_out"])}
        if case["save"]:
            out["z"] = new(M, case["n_out"])
        for g0, g1, a, e in _blocks(s):
            x = s["x"].double() if case["shared"] else s["x"][a:e].double().view(g1 - g0, (e - a) // (g1 - g0), -1)
            z = torch.matmul(x, s["w"][g0:g1].double().transpose(1, 2).contiguous())
            z = (z + s["b"][g0:g1].double().unsqueeze(1)).view(e - a, -1)
            y = _exact_act(z, act)[0]
            out["y"][a:e] = y if s["r"] is None else y + s["r"][a:e].double()
            if case["save"]:
                out["z"][a:e] = z
        return out
    if op == "linear_grad":
        out = {"dw": new(G, case["n_out"], case["n_in"]).zero_(), "db": new(G, case["n_out"]).zero_()}
        if not case["shared"]:
            out["dx"] = new(M, case["n_in"])
        for g0, g1, a, e in _blocks(s):
            n, k = (e - a) // (g1 - g0), g1 - g0
            d = s["dy"][a:e].double()
            if act != "none":
                d = d * _exact_act(s["z"][a:e].double(), act)[1]
            d = d.view(k, n, -1)
            x = s["x"].double() if case["shared"] else s["x"][a:e].double().view(k, n, -1)
            out["dw"][g0:g1] = torch.matmul(d.transpose(1, 2).contiguous(), x)
            out["db"][g0:g1] = d.sum(1)
            if not case["shared"]:
                out["dx"][a:e] = torch.matmul(d, s["w"][g0:g1].double()).view(e - a, -1)
        return out
    if op in ("layernorm", "layernorm_grad"):
        D = case["n_in"]
        out = ({"y": new(M, D), "mean": new(M), "rstd": new(M)} if op == "layernorm" else
               {"dx": new(M, D), "dgamma": new(G, D).zero_(), "dbeta": new(G, D).zero_()})
        for g0, g1, a, e in _blocks(s):
            k = g1 - g0
            x = s["x"][a:e].double().view(k, (e - a) // k, D)
            gamma = s["gamma"][g0:g1].double().unsqueeze(1)
            if op == "layernorm":
                mean = x.sum(2) / D
                rstd = ((x - mean.unsqueeze(2)).pow(2).sum(2) / D + EPS).pow(-0.5)
                y = (x - mean.unsqueeze(2)) * rstd.unsqueeze(2) * gamma + s["beta"][g0:g1].double().unsqueeze(1)
                out["y"][a:e], out["mean"][a:e], out["rstd"][a:e] = y.view(-1, D), mean.view(-1), rstd.view(-1)
                continue
            rstd = s["rstd"][a:e].double().view(k, -1, 1)
            xh = (x - s["mean"][a:e].double().view(k, -1, 1)) * rstd
            dy = s["dy"][a:e].double().view_as(x)
            p = dy * gamma
            dx = (p - p.sum(2, keepdim=True) / D - xh * ((p * xh).sum(2, keepdim=True) / D)) * rstd
            out["dx"][a:e] = dx.view(-1, D)
            out["dgamma"][g0:g1], out["dbeta"][g0:g1] = (dy * xh).sum(1), dy.sum(1)
        return out
    C = case["n_in"]
    out = {"fit": new(G), "dz": new(M, C)}
    for g0, g1, a, e in _blocks(s):
        k = g1 - g0
        logp = torch.log_softmax(s["logits"][a:e].double(), 1).view(k, -1, C)
        lab = s["labels"].view(1, -1).expand(k, -1) if case["shared"] else s["labels"][a:e].view(k, -1)
        hot = torch.arange(C, device=DEV) == lab.unsqueeze(2)
        counted = hot.any(2, keepdim=True).double()
        n = counted.sum(1, keepdim=True)
        out["fit"][g0:g1] = -torch.where(hot, logp, torch.zeros_like(logp)).sum((1, 2)) / n.view(-1)
        out["dz"][a:e] = ((logp.exp() - hot.double()) * counted / n).view(-1, C)
    return out
