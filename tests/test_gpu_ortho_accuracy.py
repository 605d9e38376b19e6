"""How exact the products of matrices of more than 64 directions are: against 64 bits, beside the same formula in 32 bits.

`plain` computes the formula in 32 bits on the CPU; `e32` is its distance from 64 bits.  The kernels hold X in two fp16
halves: a half rounds to 11 bits, so what two leave out is on average 1.5 times what 24 bits leave out (the second half's own
exponent varies: sqrt(1/2 + 1/16 + 1/128 + ...) of 2^-23 against 2^-24).  Their sums are 32-bit sums.  So their distance
is at most 1.6 e32, with 2^-21 for where the formula in 32 bits happens to be exact.  Rounding to the output's type
adds what it adds to the exact result, within a tenth (sums over some 1e5 values)."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
COEF = (3.4445, -4.7750, 2.0315)


def plain(G, steps, coef, T):
    X = G.double().cpu()
    tall = X.shape[0] > X.shape[1]
    X = X.t().contiguous() if tall else X
    X = (X / (X.norm() + 1e-7)).to(T)
    for k in range(steps):
        a, b, c = coef[k] if hasattr(coef[0], "__len__") else coef
        A = X @ X.t().contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return (X.t() if tall else X).double()


def matrix(kind, m, n):
    g = torch.Generator().manual_seed(m * 31 + n)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    k = min(m, n)
    return {"gauss": lambda: r(m, n), "rank 1": lambda: r(m, 1) @ r(1, n), "rank 8 + noise": lambda: r(m, 8) @ r(8, n) + 0.01 * r(m, n),
            "rank 8 + 1e-4": lambda: r(m, 8) @ r(8, n) + 1e-4 * r(m, n),
            "fall": lambda: (r(m, k) * torch.logspace(0, -4, k)) @ r(k, n),
            "equal": lambda: torch.linalg.qr(r(n, m))[0].t() if m <= n else torch.linalg.qr(r(m, n))[0],
            "identity": lambda: torch.eye(m, n)}[kind]().contiguous()


def norm(x):
    return float(x.norm())


def check(G, steps, coef, got, say):
    want = plain(G, steps, coef, torch.float64)
    e32 = norm(plain(G, steps, coef, torch.float32) - want)
    rounding = norm(want.to(G.dtype).double() - want)
    err = norm(got.double().cpu() - want)
    limit = 1.1 * rounding + 1.6 * e32 + 2.0 ** -21 * norm(want)
    print(f"[orth] {say} err {err / norm(want):.2e} of {limit / norm(want):.2e} (32 bits {e32 / norm(want):.1e}, "
          f"rounding {rounding / norm(want):.1e})", flush=True)
    assert err <= limit


SPECTRA = ["gauss", "rank 1", "rank 8 + noise", "rank 8 + 1e-4", "fall", "equal", "identity"]


@pytest.mark.parametrize("m,n", [(300, 400), (700, 512), (1024, 1024)])
@pytest.mark.parametrize("kind", SPECTRA)
def test_spectra_bf16(kind, m, n):
    G = matrix(kind, m, n).to(torch.bfloat16).to(DEV)
    check(G, 5, COEF, bh.orthogonalise(G), f"{kind} {m}x{n} bf16")


STEPS = [(1, COEF), (2, COEF), (12, COEF), (8, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0)),
         (3, [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)])]


@pytest.mark.parametrize("steps,coef", STEPS)
@pytest.mark.parametrize("kind", ["gauss", "equal"])
def test_steps_and_coefficients_bf16(kind, steps, coef):
    G = matrix(kind, 300, 400).to(torch.bfloat16).to(DEV)
    check(G, steps, coef, bh.orthogonalise(G, steps=steps, coefficients=coef), f"{kind} {steps} steps bf16")


def test_batch_nonfinite_strides_and_graph_bf16():
    m, n = 260, 310
    G = torch.stack([matrix(k, m, n) for k in ("gauss", "equal", "fall")]).to(torch.bfloat16).to(DEV)
    O = bh.orthogonalise(G)
    for k in range(3):
        check(G[k], 5, COEF, O[k], f"batch {k} bf16")
        assert torch.equal(O[k], bh.orthogonalise(G[k]))
    buf = torch.full((3, m + 1, n + 3), float("nan"), dtype=torch.bfloat16, device=DEV)
    buf[:, :m, :n] = G
    out = torch.full((3, m, n + 1), 42.0, dtype=torch.bfloat16, device=DEV)
    assert torch.equal(bh.orthogonalise(buf[:, :m, :n], out=out[:, :, :n]), O) and bool((out[:, :, n:] == 42.0).all())
    ws = torch.empty(bh.orthogonalise_workspace_size(3, m, n), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = bh.orthogonalise(G, workspace=ws)
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, O)
        bh.orthogonalise(O, workspace=ws)  # eager work on the same workspace
        torch.cuda.synchronize()
    G[0, 5, 7], G[2, 100, 200], G[1] = float("nan"), float("inf"), 0.0
    bad = bh.orthogonalise(G, workspace=ws)
    assert bool(torch.isnan(bad[0]).all()) and bool(torch.isnan(bad[2]).all()) and bool((bad[1] == 0).all())


def in_order(P, Q):
    """P Q^T in 32 bits, term by term in one order: sums that no machine's library changes."""
    acc = torch.zeros(P.shape[0], Q.shape[0], device=P.device)
    for k in range(P.shape[1]):
        acc = torch.addr(acc, P[:, k], Q[:, k])
    return acc


def plain_in_order(G, steps, coef):
    X = G.double().t().contiguous() if G.shape[0] > G.shape[1] else G.double()
    X = (X / (X.norm() + 1e-7)).float()
    for k in range(steps):
        a, b, c = coef[k] if hasattr(coef[0], "__len__") else coef
        A = in_order(X, X)
        X = a * X + in_order(b * A + c * in_order(A, A), X.t().contiguous())
    return (X.t() if G.shape[0] > G.shape[1] else X).double().cpu()


def check_in_order(G, steps, coef, got, say):
    """As check, with the formula in 32 bits computed term by term: a library's order of sums depends on the machine."""
    want = plain(G, steps, coef, torch.float64)
    e32 = norm(plain_in_order(G, steps, coef) - want)
    rounding = norm(want.to(G.dtype).double() - want)
    err = norm(got.double().cpu() - want)
    limit = 1.1 * rounding + 1.6 * e32 + 2.0 ** -21 * norm(want)
    print(f"[orth] {say} err {err / norm(want):.2e} of {limit / norm(want):.2e} (32 bits {e32 / norm(want):.1e}, "
          f"rounding {rounding / norm(want):.1e})", flush=True)
    assert err <= limit


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("m,n", [(130, 200), (400, 300), (1024, 1030)])
@pytest.mark.parametrize("kind", SPECTRA)
def test_spectra_as_the_formula_in_32_bits(kind, m, n, dtype):
    G = matrix(kind, m, n).to(dtype).to(DEV)
    check_in_order(G, 5, COEF, bh.orthogonalise(G), f"{kind} {m}x{n} {dtype}")


@pytest.mark.parametrize("steps,coef", STEPS)
@pytest.mark.parametrize("kind", ["gauss", "equal", "rank 8 + noise"])
def test_steps_as_the_formula_in_32_bits(kind, steps, coef):
    G = matrix(kind, 200, 130).to(DEV)
    check_in_order(G, steps, coef, bh.orthogonalise(G, steps=steps, coefficients=coef), f"{kind} {steps} steps fp32")
