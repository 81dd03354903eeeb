"""A population of networks: OpenES on their weights, then gradient descent of the best.

Every individual is a classifier 17-32-32-6 (tanh, a layer norm before the
second layer) whose parameters are one row of the population.  The evolution
draws antithetic perturbations (evox_fill_normal), evaluates all networks on
one batch of observations (evox_linear, evox_layernorm, evox_xent: the fitness
is each network's cross-entropy) and moves the center along the rank-weighted
sum of the perturbations (evox_sgemm).  The refinement takes the best networks
of the last generation and trains each by its own gradient, on a ragged share
of the data (the *_grad calls; a network's gradient is a row of a matrix like
the population).

    python examples/population_of_networks.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2301_12457_amd as evox

SIZES = (17, 32, 32, 6)


class Networks:
    """The layers of the networks whose parameters are the rows of X[N, ldx]."""

    def __init__(self, sizes=SIZES):
        n0, n1, n2, n3 = sizes
        self.sizes, self.at, self.D = sizes, {}, 0
        for name, shape in (("w1", (n1, n0)), ("b1", (n1,)), ("gamma", (n1,)), ("beta", (n1,)), ("w2", (n2, n1)),
                            ("b2", (n2,)), ("w3", (n3, n2)), ("b3", (n3,))):
            size = shape[0] if len(shape) == 1 else shape[0] * shape[1]
            self.at[name] = (self.D, size, shape)
            self.D += size

    def views(self, X):
        """The parameters by name, as views of the rows of X."""
        out = {}
        for name, (a, size, shape) in self.at.items():
            v = X[:, a:a + size]
            out[name] = v.unflatten(1, shape) if len(shape) == 2 else v
        return out

    def start(self, device):
        """A center: weights by their fan-in, gains of one."""
        theta = torch.zeros(1, evox.pitch(self.D, evox.ES), device=device)
        p = self.views(theta)
        for i, w in enumerate(("w1", "w2", "w3")):
            p[w].normal_(0.0, self.sizes[i] ** -0.5)
        p["gamma"].fill_(1.0)
        return theta

    def forward(self, X, obs, rows, off=None, keep=False):
        """Logits [rows, classes] of the networks on the observations (shared by
        them, or their own rows by off), with what the gradient needs."""
        p, n1, n2, n3 = self.views(X), *self.sizes[1:]
        new = lambda n: torch.empty(rows, n, device=X.device)
        s = {"obs": obs, "off": off, "h1": new(n1), "z1": new(n1) if keep else None, "u": new(n1), "h2": new(n2),
             "z2": new(n2) if keep else None, "mean": torch.empty(rows, device=X.device),
             "rstd": torch.empty(rows, device=X.device), "logits": new(n3)}
        evox.evox_linear(obs, p["w1"], s["h1"], b=p["b1"], z=s["z1"], off=off, act=evox.ACT_TANH)
        evox.evox_layernorm(s["h1"], p["gamma"], p["beta"], s["u"], mean=s["mean"], rstd=s["rstd"], off=off)
        # the second layer adds its input back: a residual
        evox.evox_linear(s["u"], p["w2"], s["h2"], b=p["b2"], r=s["u"] if n1 == n2 else None, z=s["z2"], off=off,
                         act=evox.ACT_TANH)
        evox.evox_linear(s["h2"], p["w3"], s["logits"], b=p["b3"], off=off)
        return s

    def backward(self, X, s, dlogits):
        """Every network's gradient, as rows like X's."""
        p, grad, off = self.views(X), torch.zeros_like(X), s["off"]
        d = self.views(grad)
        dh2, du, dh1 = torch.empty_like(s["h2"]), torch.empty_like(s["u"]), torch.empty_like(s["h1"])
        evox.evox_linear_grad(s["h2"], p["w3"], dlogits, dx=dh2, dw=d["w3"], db=d["b3"], off=off)
        evox.evox_linear_grad(s["u"], p["w2"], dh2, z=s["z2"], dx=du, dw=d["w2"], db=d["b2"], off=off,
                              act=evox.ACT_TANH)
        if self.sizes[1] == self.sizes[2]:
            du += dh2  # the residual's gradient
        evox.evox_layernorm_grad(s["h1"], p["gamma"], s["mean"], s["rstd"], du, dh1, d["gamma"], d["beta"], off=off)
        evox.evox_linear_grad(s["obs"], p["w1"], dh1, z=s["z1"], dw=d["w1"], db=d["b1"], off=off, act=evox.ACT_TANH)
        return grad


def data(n, device, seed):
    """Observations and the classes that a random linear teacher gives them."""
    g = torch.Generator(device=device).manual_seed(seed)
    teacher = torch.randn(SIZES[0], SIZES[-1], generator=torch.Generator(device=device).manual_seed(99), device=device)
    obs = torch.randn(n, SIZES[0], generator=g, device=device)
    return obs, (obs @ teacher).argmax(1).int()


def evolve(net, theta, generations=60, N=1024, batch=64, sigma=0.05, lr=0.25, seed=1):
    """OpenES: the center after these generations, the last population, the best fitness per generation."""
    device, ldx = theta.device, theta.shape[1]
    eps = torch.empty(N // 2, ldx, device=device)
    fit, history = torch.empty(N, device=device), []
    for t in range(generations):
        obs, labels = data(batch, device, seed * 1000 + t)
        evox.evox_fill_normal(seed * 1000 + t, N // 2, net.D, ldx, 0.0, 1.0, eps)
        X = torch.cat([theta + sigma * eps, theta - sigma * eps])
        evox.evox_xent(net.forward(X, obs, N * batch)["logits"], labels, fit)
        rank = fit.argsort().argsort().float() / (N - 1) - 0.5
        u = (rank[:N // 2] - rank[N // 2:]).reshape(-1, 1)
        u4 = torch.zeros(N // 2, 4, device=device)
        u4[:, :1] = u
        step = torch.empty(4, ldx, device=device)
        evox.evox_sgemm(u4, eps, step, trans_a=True, alpha=1.0 / (N * sigma))
        theta = theta - lr * step[:1]
        history.append(fit.min())
    return theta, X, fit, [float(h) for h in history]


def refine(net, X, steps=40, rows=4096, lr=0.3, seed=7):
    """Gradient descent of every network on its own share of the data."""
    G, device = X.shape[0], X.device
    obs, labels = data(rows, device, seed)
    cut = torch.sort(torch.randint(1, rows, (G - 1,), generator=torch.Generator().manual_seed(seed))).values
    off = torch.cat([torch.zeros(1), cut, torch.tensor([rows])]).int().to(device)
    fit, dlogits, history = torch.empty(G, device=device), torch.empty(rows, SIZES[-1], device=device), []
    for _ in range(steps):
        s = net.forward(X, obs, rows, off=off, keep=True)
        evox.evox_xent(s["logits"], labels, fit, dz=dlogits, off=off)
        X = X - lr * net.backward(X, s, dlogits)
        history.append(fit.nanmean())
    return X, [float(h) for h in history]


def main():
    torch.manual_seed(0)
    net = Networks()
    theta, X, fit, best = evolve(net, net.start("cuda"))
    print(f"{net.D} parameters; OpenES: best fitness {best[0]:.4f} -> {best[-1]:.4f}")
    top = X[fit.argsort()[:16]].contiguous()
    top, mean = refine(net, top)
    print(f"16 best by gradient: mean fitness {mean[0]:.4f} -> {mean[-1]:.4f}")
    return best, mean


if __name__ == "__main__":
    main()
