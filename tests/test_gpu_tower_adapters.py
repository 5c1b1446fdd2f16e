"""The operators together, as examples/tower_adapters.py uses them: the example runs, and its gradients are those of the same tower in 64 bits."""
import importlib.util
import os
import sys

import pytest
import torch

from philox import factor, kept

pytestmark = pytest.mark.gpu


def load():
    root = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
    if root not in sys.path:
        sys.path.insert(0, root)
    spec = importlib.util.spec_from_file_location("tower_adapters", os.path.join(root, "tower_adapters.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_runs():
    first, last, found = load().main(steps=3, tokens=50, n=1000, collections=3, batch=128)
    assert first > 0 and last > 0 and len(found) == 3 and all(0 <= f <= 1 for f in found)


def test_gradients():
    """Against autograd in 64 bits through the tower with the same masks and the same rounded weights.  What the calls round to bfloat16 (2^-9 of each value; h, y, z's
    gradient, the adapters and their products' results) and to 8 bits (E4M3 2^-4, E5M2 2^-3 of a value) are independent roundings, whose part in a sum of N terms grows with
    sqrt(N) while the sum of magnitudes grows with N: the gradients as a whole are off by at most the largest single rounding of their factors, 2^-3 + 2^-4."""
    tower = load().SharedTower(40, 256, 96, 3, 8, 5, torch.device("cuda:0"))
    dev = tower.state.device
    g = torch.Generator(device=dev).manual_seed(1)
    tower.p["b"] = torch.randn(tower.p["b"].shape, generator=g, device=dev) * 0.2
    n = 300
    ids = torch.randint(0, 40, (n,), generator=g, device=dev)
    which = torch.randint(-1, 3, (n,), generator=g, device=dev)
    dz = torch.randn((n, 96), generator=g, device=dev)
    z, back = tower.forward(ids, which, train=True)
    grads = tower.backward(dz, back)
    par = {k: (v.bfloat16() if k in "ab" else v).double().requires_grad_() for k, v in tower.p.items()}
    w = (tower.w[0].double().view(96, 2, 128) * tower.w[1].double()[:, :, None]).view(96, 256)
    m0, m1 = (kept(range(n), 256, tower.rate, 5, 0, layer).to(dev).double() * factor(tower.rate) for layer in (0, 1))
    h = par["table"][ids] * tower.scale * m0
    y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * par["norm"]
    own = which.clamp(min=0)
    t = ((y * m1)[:, None, :] @ par["a"][own].transpose(1, 2)) * 2.0
    z64 = y @ w.t() + torch.where((which >= 0)[:, None], (t @ par["b"][own])[:, 0], 0.0)
    assert float((z.double() - z64.detach()).norm() / z64.detach().norm()) < 2 ** -4
    z64.backward(dz.double())
    for k, got in grads.items():
        ref = par[k].grad
        assert got.shape == ref.shape and float((got.double() - ref).norm() / ref.norm()) < 2 ** -3 + 2 ** -4, k
    # the adapters' own gradients take no 8-bit products: bfloat16 roundings of y, dz, a and b alone, four factors
    for k in "ab":
        assert float((grads[k].double() - par[k].grad).norm() / par[k].grad.norm()) < 4 * 2 ** -8, k
