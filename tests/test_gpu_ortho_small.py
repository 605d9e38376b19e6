"""Matrices far below eps, and coefficients that shrink: X is small against one, and keeps its digits.

Where |U| is far below eps, X = U / (|U| + eps) is too, and the steps multiply it by a.  Tolerance: a product's operands
of 22 bits and sums of 32, 2^-21 of the result's size a step, and five steps of it; then the output's rounding."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
COEF = (3.4445, -4.7750, 2.0315)
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def plain(G, steps=5, coef=COEF, eps=1e-7):
    X = G.double().cpu()
    tall = X.shape[0] > X.shape[1]
    X = X.t().contiguous() if tall else X
    X = X / (X.norm() + eps)
    a, b, c = coef
    for _ in range(steps):
        A = X @ X.t().contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.t() if tall else X


def rel(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


def gauss(m, n, seed=1):
    return torch.randn(m, n, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(130, 200), (400, 300), (40, 60)])
@pytest.mark.parametrize("scale", [1e-8, 1e-10, 1e-12, 1e-14, 1e-16, 1e-18, 1e-22, 1e-28])
def test_far_below_eps(scale, shape, dtype):
    G = (gauss(*shape) * scale).to(dtype).to(DEV)
    r = rel(bh.orthogonalise(G), plain(G))
    print(f"[orth] {shape} {scale} {dtype} {r:.1e}", flush=True)
    assert r <= 5 * 2.0 ** -21 + HALF[dtype]


def test_each_matrix_of_a_batch_for_itself():
    G = torch.stack([gauss(130, 90, k) * s for k, s in enumerate((1.0, 1e-15, 0.0, 1e-9, 1e4))]).to(DEV)
    O = bh.orthogonalise(G)
    assert all(torch.equal(O[k], bh.orthogonalise(G[k])) for k in range(5))
    assert max(rel(O[k], plain(G[k])) for k in (0, 1, 3, 4)) <= 5 * 2.0 ** -21 + 2.0 ** -24 and bool((O[2] == 0).all())


@pytest.mark.parametrize("eps", [1e-3, 1.0, 100.0])
def test_large_eps(eps):
    G = (1e-6 * gauss(200, 150)).to(DEV)
    assert rel(bh.orthogonalise(G, eps=eps), plain(G, eps=eps)) <= 5 * 2.0 ** -21 + 2.0 ** -24


def test_momentum_step_far_below_eps():
    G = (1e-17 * gauss(150, 140)).to(DEV)
    W, M = torch.zeros(150, 140, device=DEV), torch.zeros(150, 140, device=DEV)
    bh.muon_step(W, G, M, 1.0, 0.0, nesterov=False, scale=1.0)
    assert rel(-W, plain(G)) <= 5 * 2.0 ** -21 + 2.0 ** -24


@pytest.mark.parametrize("steps,coef", [(20, (0.5, 0.0, 0.0)), (16, (0.4, -0.1, 0.02)), (32, (0.3, 0.2, 0.0))])
@pytest.mark.parametrize("shape", [(130, 200), (40, 60)])
def test_coefficients_that_shrink(shape, steps, coef):
    G = gauss(*shape).to(DEV)
    r = rel(bh.orthogonalise(G, steps=steps, coefficients=coef), plain(G, steps, coef))
    print(f"[orth] {shape} {steps} steps {coef} {r:.1e}", flush=True)
    assert r <= steps * 2.0 ** -21
