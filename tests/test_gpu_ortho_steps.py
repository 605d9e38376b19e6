"""Newton-Schulz steps of matrices of few directions and of low rank, against the recurrence on X itself in 64 bits.

Inputs here are of rank 1 to 5, rounded to their type, with rows that are equal, and gaussian ones.

Tolerances: both sides compute in 64 bits.  Their rounding, some 2^-50, grows with the input's own smallest directions,
which for a product rounded to 24 bits lie at 1e-9 of its norm or above: 2^-50 / 1e-9 = 1e-6 of these, and ten times that for
the spread of directions.  Equal rows stay equal where every row's sums run in the same order, as they do on both
sides.  Then the output's own rounding, half a unit in its last place at most."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
COEF = (3.4445, -4.7750, 2.0315)
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def by_rows(P, Q):
    """P Q with every row's sums in one order."""
    return torch.stack([(p[:, None] * Q).sum(0) for p in P])


def on_x(G, steps, coef=COEF, eps=1e-7):
    G = G.double().cpu()
    X = G.t().contiguous() if G.shape[0] > G.shape[1] else G
    X = X / (X.square().sum().sqrt() + eps)
    for k in range(steps):
        a, b, c = coef[k] if hasattr(coef[0], "__len__") else coef
        A = torch.stack([(x * X).sum(1) for x in X])
        X = a * X + by_rows(b * A + c * by_rows(A, A), X)
    return X.t() if G.shape[0] > G.shape[1] else X


def matrix(kind, rows, cols, dtype):
    g = torch.Generator().manual_seed(rows * 7919 + cols)
    if kind == "ones":
        G = torch.ones(rows, cols)
    elif kind == "equal rows":
        G = torch.randn(1, cols, generator=g).expand(rows, cols)
    elif kind == "gauss":
        G = torch.randn(rows, cols, generator=g)
    else:
        G = torch.randn(rows, kind, generator=g) @ torch.randn(kind, cols, generator=g)
    return G.to(dtype).to(DEV)


def rel(got, want):
    got = got.double().cpu()
    return float((got - want).norm() / want.norm())


# of one launch's size and of two launches', wide and tall
CASES = [(1, 32, 100), (5, 50, 256), (3, 40, 1500), (2, 700, 48), ("ones", 64, 64), ("ones", 16, 5000), ("equal rows", 2, 128),
         ("equal rows", 9, 2500), ("gauss", 20, 300), ("gauss", 64, 65)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("steps", [6, 7, 8, 9])
@pytest.mark.parametrize("kind,rows,cols", CASES)
def test_steps_of_low_rank(kind, rows, cols, steps, dtype):
    G = matrix(kind, rows, cols, dtype)
    want = on_x(G, steps)
    got = bh.orthogonalise(G, steps=steps)
    print(f"[orth] {kind} {rows}x{cols} {steps} steps {dtype} {rel(got, want):.1e}", flush=True)
    assert bool(torch.isfinite(got).all())
    assert rel(got, want) <= 1e-5 + HALF[dtype]


@pytest.mark.parametrize("steps", [5, 9])
@pytest.mark.parametrize("rows,cols", [(20, 300), (64, 100), (33, 900)])
def test_coefficients_are_taken_as_given(rows, cols, steps):
    """Coefficients are doubles: in fp32 (1e-8 of them) their rounding would be three times the output's."""
    G = matrix("gauss", rows, cols, torch.float32)
    r = rel(bh.orthogonalise(G, steps=steps), on_x(G, steps))
    print(f"[orth] {rows}x{cols} {steps} steps {r:.1e}", flush=True)
    assert r <= 2.0 ** -24 + 2.0 ** -27


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("steps", [10, 11, 12, 14, 16, 20, 32])
@pytest.mark.parametrize("kind,rows,cols", CASES)
def test_many_steps_of_low_rank(kind, rows, cols, steps, dtype):
    """A direction that the input lacks has an eigenvalue of A = X X^T that is zero but for rounding, of either sign.  On X
    it grows by a a step and stays bounded; on A alone it would grow by a^2, and below zero without end."""
    G = matrix(kind, rows, cols, dtype)
    want = on_x(G, steps)
    got = bh.orthogonalise(G, steps=steps)
    print(f"[orth] {kind} {rows}x{cols} {steps} steps {dtype} {rel(got, want):.1e}", flush=True)
    assert bool(torch.isfinite(got).all())
    assert rel(got, want) <= 1e-5 + HALF[dtype]


@pytest.mark.parametrize("rows,cols", [(12, 70), (12, 1100), (1100, 12)])
def test_a_batch_in_place_with_strides_and_the_momentum_step(rows, cols):
    G = torch.stack([matrix(k, rows, cols, torch.float32) for k in (1, 2, "gauss")])
    want = [on_x(g, 20) for g in G]
    alone = [bh.orthogonalise(g, steps=20) for g in G]
    buf = torch.full((3, rows + 1, cols + 3), float("nan"), device=DEV)
    view = buf[:, :rows, :cols]
    view.copy_(G)
    assert bh.orthogonalise(view, steps=20, out=view) is view
    assert all(torch.equal(view[k], alone[k]) for k in range(3)) and bool(torch.isnan(buf[:, rows:]).all())
    assert max(rel(view[k], want[k]) for k in range(3)) <= 1e-5 + 2.0 ** -24
    # the momentum is updated once, and the weights by the whole step
    W, M = 0.1 * torch.randn(3, rows, cols, device=DEV), torch.zeros(3, rows, cols, device=DEV)
    before = W.double()
    bh.muon_step(W, G, M, 0.5, 0.9, nesterov=False, weight_decay=0.1, scale=1.25, steps=20)
    assert torch.equal(M, G)
    step = (before * (1 - 0.05) - W.double()) / (0.5 * 1.25)
    assert max(rel(step[k], want[k]) for k in range(3)) <= 1e-4  # weights of 0.1 in 24 bits, taken apart again


def test_many_steps_replay_in_a_graph():
    G = matrix(3, 30, 400, torch.float32)
    ws = torch.empty(bh.orthogonalise_workspace_size(1, 30, 400), dtype=torch.uint8, device=DEV)
    want = bh.orthogonalise(G, steps=16, workspace=ws).clone()
    out = torch.zeros_like(G)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bh.orthogonalise(G, steps=16, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        bh.orthogonalise(want, steps=3, workspace=ws)  # eager work on the same workspace
        torch.cuda.synchronize()


def test_zero_and_nonfinite_matrices_of_many_steps():
    G = torch.zeros((3, 10, 80), device=DEV)
    G[1] = matrix("gauss", 10, 80, torch.float32)
    G[2] = G[1]
    G[2, 3, 4] = float("nan")
    O = bh.orthogonalise(G, steps=20)
    assert bool((O[0] == 0).all()) and bool(torch.isnan(O[2]).all()) and rel(O[1], on_x(G[1], 20)) <= 1e-5
    G[2, 3, 4] = float("inf")
    assert bool(torch.isnan(bh.orthogonalise(G, steps=20)[2]).all())
