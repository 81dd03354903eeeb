"""The example of a population of networks learns by both of its ways, and its
whole gradient (through all layers, the norm, the residual and the loss) agrees
with central differences of the fitness."""
import os
import sys

import pytest
import torch

from conftest import ROOT

sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


def test_example_learns(evox_gpu):
    import population_of_networks as ex
    best, mean = ex.main()
    assert best[-1] < 0.6 * best[0]
    assert mean[-1] < mean[0]


def test_gradient_through_the_network(evox_gpu):
    import population_of_networks as ex
    torch.manual_seed(1)
    net, G, rows = ex.Networks(), 5, 300
    X = torch.cat([net.start("cuda") for _ in range(G)])
    obs, labels = ex.data(rows, "cuda", 3)
    off = torch.tensor([0, 40, 40 + 1, 150, 200, 300], dtype=torch.int32, device="cuda")
    fit, dl = torch.empty(G, device="cuda"), torch.empty(rows, ex.SIZES[-1], device="cuda")

    def fitness(X):
        s = net.forward(X, obs, rows, off=off, keep=True)
        evox_gpu.evox_xent(s["logits"], labels, fit, dz=dl, off=off)
        return s, fit.double().clone()

    s, _ = fitness(X)
    grad = net.backward(X, s, dl.clone())[:, :net.D].double()
    u = torch.randn(G, X.shape[1], device="cuda")
    u[:, net.D:] = 0
    h = 2.0 ** -9
    diff = (fitness(X + h * u)[1] - fitness(X - h * u)[1]) / (2 * h)
    got = (grad * u[:, :net.D].double()).sum(1)
    # fitness carries about 2^-21; the second-order term is h^2 times a third
    # derivative of the order of |u|^3 = D^1.5 over the layers' fan-ins
    limit = 2.0 ** -21 / h + 0.02 * grad.norm(dim=1)
    assert ((diff - got).abs() <= limit).all(), (diff, got, limit)
