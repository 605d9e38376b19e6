"""The loss from neighbour lists and its gradient, against the formulas in 64 bits and against differences.

Tolerances: u = 2^-24.  An exponential of x = |z - top| / T is taken of an argument with three roundings (the difference, log2 e / T,
their product) and is off by 2 u itself: (4 x + 4) u of its value.  A lane adds up at most 64 terms or v / 256 (parts of 8192 values or
more), and its wave and block 10 more.  So the sum is off by (4 x + terms) u of its terms, where x is averaged with the terms'
weights."""
import math

import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def say(*a):
    print(*a, flush=True)


def case(n, v, k, dtype, seed, pad=0, teacher=torch.float32, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((n, v + pad), float("nan"), dtype=dtype)
    buf[:, :v] = (spread * torch.randn(n, v, generator=g)).to(dtype)
    idx = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(n)]) if n and k else torch.zeros(n, k)
    u = (-3.0 * torch.rand(n, k, generator=g)).to(teacher)
    return buf.to(DEV)[:, :v], idx.to(torch.int32).to(DEV), u.to(DEV)


def reference(z, idx, u, T):
    z, u = z.double().cpu() / T, u.double().cpu() / T
    v = z.shape[1]
    idx = idx.cpu().long()
    there = (idx >= 0) & (idx < v) & (u > -math.inf)
    u = torch.where(there, u, -math.inf)
    top = u.amax(1, keepdim=True) if u.shape[1] else torch.zeros(len(u), 1, dtype=torch.float64)
    x_t = torch.where(there, top - u, 0.0)
    t = torch.where(there, torch.exp(-x_t), 0.0)
    total = t.sum(1, keepdim=True)
    t = torch.where(total > 0, t / total, 0.0)
    lse = torch.logsumexp(z, 1)
    at = idx.clamp(0, v - 1)
    terms = torch.where(t > 0, t * (-x_t - total.log() - z.gather(1, at) + lse[:, None]), 0.0)
    return z, at, t, x_t, lse, terms


def terms_of(v):
    return 80.0 + v / 256


def check_forward(z, idx, u, T, got):
    loss, lse = (r.double().cpu() for r in got)
    z, at, t, x_t, e_lse, terms = reference(z, idx, u, T)
    x = z.amax(1, keepdim=True) - z
    tol_lse = U * (4 * (torch.exp(z - e_lse[:, None]) * x).nan_to_num(nan=0.0).sum(1) + terms_of(z.shape[1]))  # x e^-x: 0 at infinity
    assert got[0].dtype == got[1].dtype == torch.float32
    assert bool(((lse - e_lse).abs() <= tol_lse + U * e_lse.abs()).all())
    rel = U * (4 * x_t + 4 * (t * x_t).sum(1, keepdim=True) + 16)
    tol = (rel * terms.abs() + t * (2 * U * x_t + tol_lse[:, None])).sum(1)
    want = terms.sum(1)
    err = (loss - want).abs()
    assert bool((err <= tol + U * (want.abs() + tol)).all()), float((err - tol).max())


def check_backward(dloss, z, idx, u, lse, T, got):
    dtype = z.dtype
    z, at, t, x_t, _, _ = reference(z, idx, u, T)
    g = dloss.double().cpu()[:, None] / T
    lse = lse.double().cpu()[:, None]
    q = torch.exp(z - lse) * t.sum(1, keepdim=True).round()
    want = (g * q).scatter_add_(1, at, -g * t)
    share = U * (4 * x_t + 4 * (t * x_t).sum(1, keepdim=True) + 16) * t
    tol = (g.abs() * (q * U * (4 * (z - lse).abs() + 16)).nan_to_num(nan=0.0)).scatter_add_(1, at, g.abs() * share)
    tol = tol + HALF[dtype] * (want.abs() + tol) + TINY[dtype]
    err = (got.double().cpu() - want).abs()
    assert got.dtype == dtype and bool((err <= tol).all()), float((err / tol).max())


SIZES = [(1, 1, 1), (1, 2, 2), (5, 7, 3), (3, 64, 64), (33, 100, 10), (20, 1000, 90), (7, 2048, 30), (6, 2049, 300), (4, 5003, 257), (300, 50, 1), (9, 8192, 90),
         (3, 8193, 20), (2, 70_001, 90), (1, 300_007, 30), (2500, 2100, 5), (2, 3000, 2048)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v,k", SIZES)
def test_both_directions(n, v, k, dtype):
    for pad, teacher, T in ((0, torch.float32, 1.0), (3, dtype, 2.0), (8, torch.float32, 0.5)):
        say(f"[distil] {n} x {v}, {k} listed, pad {pad}, T {T} {dtype}")
        z, idx, u = case(n, v, k, dtype, n + v + k, pad, teacher)
        loss, lse = bh.distil_loss(z, idx, u, T)
        check_forward(z, idx, u, T, (loss, lse))
        dloss = torch.linspace(-1.0, 1.5, n, device=DEV)
        dz = bh.distil_loss_backward(dloss, z, idx, u, lse, T)
        check_backward(dloss, z, idx, u, lse, T, dz)
        again = bh.distil_loss(z, idx, u, T)
        assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
        # in place, and into rows with gaps at another alignment
        gap = torch.full((n, v + 5), 7.0, dtype=dtype, device=DEV)
        bh.distil_loss_backward(dloss, z, idx, u, lse, T, dlogits=gap[:, 1:v + 1])
        assert torch.equal(gap[:, 1:v + 1], dz) and bool((gap[:, :1] == 7).all()) and bool((gap[:, v + 1:] == 7).all())
        same = bh.distil_loss_backward(dloss, z, idx, u, lse, T, dlogits=z)
        assert same is z and torch.equal(z, dz)


def test_absent_entries():
    for t in TYPES:
        for v in (40, 3000, 20_000):
            z, idx, u = case(6, v, 12, t, v)
            idx[0, 3:], idx[1], idx[2, 0], idx[3, 5] = -1, -1, v, -(1 << 31)
            u[4, 1:], u[5] = -math.inf, -math.inf
            u[0, 3:] = float("nan")  # of what is absent nothing counts
            loss, lse = bh.distil_loss(z, idx, u)
            dloss = torch.ones(6, device=DEV)
            u2 = torch.nan_to_num(u, nan=0.0, neginf=-math.inf)
            check_forward(z, idx, u2, 1.0, (loss, lse))
            dz = bh.distil_loss_backward(dloss, z, idx, u, lse)
            check_backward(dloss, z, idx, u2, lse, 1.0, dz)
            assert loss[1] == 0 and loss[5] == 0 and not dz[1].any() and not dz[5].any()


def test_no_list_and_no_rows():
    z, idx, u = case(5, 300, 0, torch.float32, 1)
    loss, lse = bh.distil_loss(z, idx, u)
    assert not loss.any() and not bh.distil_loss_backward(loss, z, idx, u, lse).any()
    z, idx, u = case(0, 300, 4, torch.float32, 1)
    loss, lse = bh.distil_loss(z, idx, u)
    assert loss.shape == (0,) and bh.distil_loss_backward(loss, z, idx, u, lse).shape == (0, 300)


def test_a_class_listed_more_than_once():
    for v in (10, 5000, 30_000):
        z, idx, u = case(4, v, 9, torch.float32, v)
        idx[0], idx[1, 4:], idx[2, 1] = 3, 7, int(idx[2, 0])
        loss, lse = bh.distil_loss(z, idx, u)
        check_forward(z, idx, u, 1.0, (loss, lse))
        dloss = torch.ones(4, device=DEV)
        dz = bh.distil_loss_backward(dloss, z, idx, u, lse)
        check_backward(dloss, z, idx, u, lse, 1.0, dz)
        assert torch.equal(dz, bh.distil_loss_backward(dloss, z, idx, u, lse))


def test_masked_and_extreme_logits():
    """Classes that are masked out by minus infinity or the type's lowest value; logits that all are far from zero."""
    for t in TYPES:
        for v in (50, 3000, 20_000):
            z, idx, u = case(5, v, 6, t, v)
            listed = idx[0].long()
            mask = torch.ones(v, dtype=torch.bool, device=DEV)
            mask[listed] = False
            z[0, mask] = -math.inf
            z[1, : v // 2] = -math.inf
            idx[1] = torch.arange(v - 6, v, dtype=torch.int32, device=DEV)
            z[2, : v // 2] = torch.finfo(t).min
            idx[2] = idx[1]
            z[3] += 3e4 if t != torch.float16 else 1e3
            loss, lse = bh.distil_loss(z, idx, u)
            exact = [r for r in range(5) if r != 3]
            check_forward(z[exact], idx[exact], u[exact], 1.0, (loss[exact], lse[exact]))
            dloss = torch.ones(5, device=DEV)
            dz = bh.distil_loss_backward(dloss, z, idx, u, lse)
            check_backward(dloss, z, idx, u, lse, 1.0, dz)
            assert bool(loss.isfinite().all())
            # a listed class without a probability: an infinite loss, a finite gradient
            z[4, idx[4, 0].long()] = -math.inf
            loss, lse = bh.distil_loss(z, idx, u)
            assert loss[4] == math.inf and bool(bh.distil_loss_backward(dloss, z, idx, u, lse)[4].isfinite().all())


def test_nan_stays_in_its_row():
    for v in (50, 3000, 20_000):
        z, idx, u = case(5, v, 6, torch.float32, v)
        want, lse = bh.distil_loss(z, idx, u)
        z[1, v // 3], z[3, 1] = float("nan"), float("inf")
        got, lse2 = bh.distil_loss(z, idx, u)
        assert bool(got[[1, 3]].isnan().all()) and torch.equal(got[[0, 2, 4]], want[[0, 2, 4]]) and torch.equal(lse[[0, 2, 4]], lse2[[0, 2, 4]])


def test_gradient_against_differences():
    n, v, k, T = 3, 12, 4, 1.5
    z, idx, u = case(n, v, k, torch.float32, 5)
    z = z.clone().requires_grad_()
    w = torch.tensor([1.0, -0.5, 2.0], device=DEV)
    (bh.distil_loss(z, idx, u, T)[0] * w).sum().backward()
    base, step = z.detach().double().cpu(), 1e-5
    for at in range(n * v):
        ends = []
        for sign in (1, -1):
            moved = base.clone()
            moved.view(-1)[at] += sign * step
            ends.append(float((reference(moved, idx, u, T)[5].sum(1) * w.double().cpu()).sum()))
        assert abs((ends[0] - ends[1]) / (2 * step) - float(z.grad.view(-1)[at])) <= 1e-6


def test_in_torch_graph():
    z, idx, u = case(40, 500, 20, torch.bfloat16, 3)
    z = z.clone().requires_grad_()
    loss, lse = bh.distil_loss(z, idx, u)
    assert loss.requires_grad and not lse.requires_grad
    loss.mean().backward()
    want = bh.distil_loss_backward(torch.full((40,), 1 / 40, device=DEV), z.detach(), idx, u, lse)
    assert torch.equal(z.grad, want)
    with pytest.raises(ValueError, match="gradient"):
        bh.distil_loss(z, idx, u.requires_grad_())
    with torch.no_grad():
        assert not bh.distil_loss(z, idx, u)[0].requires_grad


def test_neighbours_of_affinities():
    """The lists that bhtsne_affinities takes: with u = -d^2 / (2 sigma^2) the teacher's shares are its p_j|i."""
    n, k = 400, 30
    x = torch.randn(n, 8, generator=torch.Generator().manual_seed(2)).to(DEV)
    d = torch.cdist(x, x)
    d.fill_diagonal_(float("inf"))
    dist, idx = torch.topk(d, k, largest=False)
    idx, dist = idx.to(torch.int32).contiguous(), dist.contiguous()
    out = bh.affinities(idx, dist, 10.0, sigma2=True)
    sigma2 = out[1].double()
    u = (-dist.double().square() / (2 * sigma2[:, None])).float()
    z = torch.zeros(n, n, device=DEV)
    loss, lse = bh.distil_loss(z, idx, u)
    # against the same q for all: log n - entropy, and the entropy of each row is log(perplexity)
    assert bool((loss.double() - (math.log(n) - math.log(10.0))).abs().max() <= 1e-4)
