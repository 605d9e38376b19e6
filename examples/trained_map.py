"""A map from features to the plane, trained with the t-SNE gradient, so that new points can be placed too.

An encoder of dense layers, each hidden one followed by a layer norm and a GELU, takes every point's features to its
place Y.  The gradient of the t-SNE cost at Y (bhtsne_gradient) goes back through it: torch does the dense products,
the library the layer norms (bhtsne_layer_norm, bhtsne_layer_norm_backward) and the steps of the weight matrices along
their orthogonalised momentum (bhtsne_muon_step).  Held-out points are then placed by the map alone.

    python examples/trained_map.py --points 4000 --steps 300
"""
import argparse
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2212_11506_amd as bh  # noqa: E402


class Map:
    """Weights W (out x in), each hidden layer with a norm's weight and bias, and the momenta of all of them."""

    def __init__(self, sizes, seed=0, device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        make = lambda o, i: torch.randn((o, i), generator=gen, device=device) / math.sqrt(i)  # noqa: E731
        self.weights = [make(o, i).requires_grad_() for i, o in zip(sizes, sizes[1:])]
        self.weights[-1].data.mul_(1e-2)  # the embedding starts small, as a free one does
        self.norms = [(torch.ones(o, device=device).requires_grad_(), torch.zeros(o, device=device).requires_grad_())
                      for o in sizes[1:-1]]
        self.momenta = [torch.zeros_like(w) for w in self.weights]

    def __call__(self, x):
        for w, (scale, shift) in zip(self.weights, self.norms):
            x = F.gelu(bh.layer_norm(x @ w.t(), scale, shift)[0])
        return x @ self.weights[-1].t()

    def step(self, learning_rate, momentum):
        with torch.no_grad():
            for w, m in zip(self.weights, self.momenta):
                bh.muon_step(w, w.grad, m, learning_rate, momentum)
                w.grad = None
            for pair in self.norms:
                for p in pair:  # vectors have no directions to make equal: a step of unit length
                    p.sub_(learning_rate * p.grad / (p.grad.norm() + 1e-12))
                    p.grad = None


def blobs(n, clusters, features, seed, device="cuda"):
    """Points of equal Gaussian clusters, and the cluster of each."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    centres = 4.0 * torch.randn((clusters, features), generator=gen, device=device)
    which = torch.randint(clusters, (n,), generator=gen, device=device)
    return centres[which] + torch.randn((n, features), generator=gen, device=device), which


def similarities(x, perplexity):
    """P of the points' nearest neighbours, brute force: the library takes neighbour lists from anywhere."""
    k = min(3 * int(perplexity), x.shape[0] - 1)
    d = torch.cdist(x, x)
    d.fill_diagonal_(float("inf"))
    dist, idx = torch.topk(d, k, largest=False)
    return bh.affinities(idx.to(torch.int32).contiguous(), dist.contiguous(), perplexity)[0]


def train(n=4000, steps=300, clusters=10, features=50, hidden=256, perplexity=30.0, seed=0, say=print):
    """(cost of the start, cost of the end, share of held-out points nearest to their own cluster's place)."""
    x, which = blobs(n + n // 4, clusters, features, seed)
    seen, new = x[:n].contiguous(), x[n:].contiguous()
    P = similarities(seen, perplexity)
    net = Map([features, hidden, hidden, 2], seed)
    ws = torch.empty(bh.workspace_size(n, P.nnz), dtype=torch.uint8, device=x.device)

    def cost():
        with torch.no_grad():
            Y = net(seen).contiguous()
        return bh.kl(Y, P, bh.z_exact(Y, workspace=ws), workspace=ws)

    first = cost()
    say(f"{n} points, {P.nnz} entries of P: KL {first:.3f} at the start")
    for it in range(steps):
        early = it < steps // 4
        Y = net(seen)
        grad, _ = bh.gradient(Y.detach().contiguous(), P, 0.5, 12.0 if early else 1.0, workspace=ws, return_z=False)
        Y.backward(grad)
        net.step(0.1 * (1.0 - it / steps) + 0.002, 0.8 if early else 0.95)
        if (it + 1) % 100 == 0:
            say(f"step {it + 1}: KL {cost():.3f}")
    last = cost()
    with torch.no_grad():
        Y, Ynew = net(seen), net(new)
        centres = torch.stack([Y[which[:n] == c].mean(0) for c in range(clusters)])
        right = (torch.cdist(Ynew, centres).argmin(1) == which[n:]).float().mean().item()
    say(f"KL {last:.3f} after {steps} steps; {100 * right:.1f} % of {n // 4} new points lie nearest to their own cluster")
    return first, last, right


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--points", type=int, default=4000)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--clusters", type=int, default=10)
    a = ap.parse_args()
    train(a.points, a.steps, a.clusters)
