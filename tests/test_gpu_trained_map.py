"""The example that trains a map runs as a user would run it: the layer norms' gradients against torch's own graph,
and a short training that lowers the cost and places points it has not seen."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("trained_map", os.path.join(ROOT, "examples", "trained_map.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_of_the_map():
    m = example()
    net = m.Map([20, 64, 32, 2], seed=3)
    x = m.blobs(500, 4, 20, 1)[0]
    r = m.blobs(500, 4, 2, 2)[0]
    net(x).backward(r)
    mine = [w.grad for w in net.weights] + [p.grad for pair in net.norms for p in pair]
    # the same map in 64 bits by torch alone
    weights = [w.detach().double().cpu().requires_grad_() for w in net.weights]
    norms = [tuple(p.detach().double().cpu().requires_grad_() for p in pair) for pair in net.norms]
    y = x.double().cpu()
    for w, (scale, shift) in zip(weights, norms):
        y = F.gelu(F.layer_norm(y @ w.t(), (w.shape[0],), scale, shift, 1e-5))
    (y @ weights[-1].t()).backward(r.double().cpu())
    want = [w.grad for w in weights] + [p.grad for pair in norms for p in pair]
    for a, b in zip(mine, want):
        # sums of 500 rows in fp32 through three layers
        assert float((a.double().cpu() - b).norm()) <= 1e-4 * float(b.norm())


def test_a_short_training_places_new_points():
    first, last, right = example().train(n=1600, steps=120, clusters=6, hidden=128, say=lambda *a: print(*a, flush=True))
    assert last < 0.6 * first and right > 0.9
