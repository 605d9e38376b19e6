"""The loss from neighbour lists where lists or logits leave the finite numbers."""
import math

import pytest
import torch

import paper_2212_11506_amd as bh
from tests.test_gpu_distil import HALF, TINY, TYPES, U, case, check_forward, reference, terms_of

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")
ROWS = [(6, 40), (6, 3000), (3, 30_000)]  # a wave's, a block's, shared out over several blocks


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", ROWS)
@pytest.mark.parametrize("k", [1, 2, 90])
def test_a_list_of_nan_is_no_empty_list(n, v, k, dtype):
    """NaN in every entry that a row has: NaN is what the loss and the listed places' gradient are, not 0."""
    k = min(k, v)
    for teacher in {dtype, torch.float32}:
        z, idx, u = case(n, v, k, dtype, n + v + k, 3, teacher)
        dloss = torch.ones(n, device=DEV)
        want, lse = bh.distil_loss(z, idx, u)
        dz = bh.distil_loss_backward(dloss, z, idx, u, lse)
        u[0] = NAN
        if k > 1:  # beside entries that are absent by either mark
            u[1], idx[1, 1:] = NAN, -1
            u[2], u[2, 1:] = NAN, -math.inf
        bad = [0, 1, 2] if k > 1 else [0]
        good = [r for r in range(n) if r not in bad]
        loss, lse2 = bh.distil_loss(z, idx, u)
        got = bh.distil_loss_backward(dloss, z, idx, u, lse)
        assert torch.equal(lse, lse2) and torch.equal(loss[good], want[good]) and torch.equal(got[good], dz[good])
        assert bool(loss[bad].isnan().all())
        for r in bad:
            listed = torch.zeros(v, dtype=torch.bool, device=DEV)
            listed[idx[r][idx[r] >= 0].long()] = True
            nan = torch.zeros(v, dtype=torch.bool, device=DEV)
            nan[idx[r][(idx[r] >= 0) & u[r].isnan()].long()] = True
            assert bool(got[r][nan].isnan().all())
            # what is not listed has its probability alone, as in any row with a list: half a step of bf16, and some u of the
            # exponential and lse, are below 2^-7; half the spacing of fp16's subnormals is 2^-25
            q = torch.exp(z[r].double() - lse[r].double())
            assert bool(((got[r].double() - q).abs() <= 2.0 ** -7 * q + 2.0 ** -24)[~listed].all())
        # through torch's graph too
        leaf = z.clone().requires_grad_()
        bh.distil_loss(leaf, idx, u)[0].sum().backward()
        assert bool(leaf.grad[0].isnan().any())


def far_rows(n, v, dtype, T, seed):
    """Rows that leave no class (the type's lowest value everywhere), nearly none, or lie as far off as the type reaches."""
    z, idx, u = case(n, v, min(v, 7), dtype, seed)
    lowest, largest = torch.finfo(dtype).min, torch.finfo(dtype).max
    z[0] = lowest
    z[1], z[1, idx[1, :3].long()] = lowest, z[1, idx[1, :3].long()]
    z[2] = largest
    if n > 3:
        z[3], z[3, idx[3, 0].long()] = lowest / 2, lowest
        z[4] = z[4] * (largest / 64)
        z[5] = z[5] * T + largest / 1024
    return z, idx, u


def shifted(z):
    """The same softmax, in 64 bits: logits less their row's largest."""
    return z.double() - z.double().amax(1, keepdim=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", ROWS)
def test_loss_of_rows_far_off(n, v, dtype):
    for T in (1.0, 0.05, 1e-6, 300.0):
        z, idx, u = far_rows(n, v, dtype, T, n + v)
        loss, _ = bh.distil_loss(z, idx, u, T)
        near = shifted(z)
        lse = torch.logsumexp(near / T, 1).float()
        # a loss beyond the largest fp32 number is rounded to infinity
        held = reference(near, idx, u, T)[5].sum(1) <= torch.finfo(torch.float32).max
        assert bool((loss.cpu()[~held] == math.inf).all())
        held = held.to(DEV)
        check_forward(near[held], idx[held], u[held], T, (loss[held], lse[held]))
    # no class at all: log v less the list's entropy
    t = torch.softmax(u[0].double(), 0)
    loss = bh.distil_loss(z, idx, u)[0]
    assert abs(float(loss[0]) - float((t * t.log()).sum()) - math.log(v)) <= 100 * 2.0 ** -24 * math.log(v)


def same(p, q):
    return torch.equal(p.isnan(), q.isnan()) and torch.equal(p.nan_to_num(nan=0.0), q.nan_to_num(nan=0.0))


def check_gradient(dloss, z, idx, u, T, got):
    """As the list's own test has it, but against the softmax itself, not the rounded lse.  q is the quotient of an exponential
    and the row's sum, which is off as the forward pass' is; where |lse| < 16 lse's rounding, 8 u, and its product with T's,
    as much again, take the sum's place.  An exponential below 2^-126 is 0."""
    dtype, v = got.dtype, z.shape[1]
    near, at, t, x_t, lse, _ = reference(shifted(z), idx, u, T)
    g = dloss.double().cpu()[:, None] / T
    q = torch.exp(near - lse[:, None]) * t.sum(1, keepdim=True).round()
    want = (g * q).scatter_add_(1, at, -g * t)
    of_sum = U * (4 * (q * -near).nan_to_num(nan=0.0).sum(1, keepdim=True) + terms_of(v))  # x e^-x: 0 at infinity
    share = U * (4 * x_t + 4 * (t * x_t).sum(1, keepdim=True) + 16) * t
    tol = (g.abs() * ((q * (U * (4 * -near + 32) + of_sum)).nan_to_num(nan=0.0) + 2.0 ** -126)).scatter_add_(1, at, g.abs() * share)
    tol = tol + HALF[dtype] * (want.abs() + tol) + TINY[dtype]
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", ROWS)
def test_gradient_of_rows_far_off(n, v, dtype):
    """The gradient through torch's graph where lse is so large that its rounding counts."""
    for T in (1.0, 0.05, 1e-6, 300.0):
        for far in (True, False):
            if far:
                z, idx, u = far_rows(n, v, dtype, T, n + v)
            else:  # any row of a head whose logits have drifted
                z, idx, u = case(n, v, min(v, 7), dtype, n + v)
                z = ((z.double() * T + torch.linspace(-1000 * T, 60_000 * min(T, 1.0), n, device=DEV)[:, None])).to(dtype)
            dloss = T * torch.linspace(-1.0, 1.5, n, device=DEV)
            leaf = z.clone().requires_grad_()
            loss, lse, kept = bh.distil_loss(leaf, idx, u, T, keep=True)
            loss.backward(dloss)
            there = z.amax(1) > -math.inf  # rows that the type holds: others are minus infinity, and NaN by the formula
            check_gradient(dloss[there], z[there], idx[there], u[there], T, leaf.grad[there])
            assert bool(leaf.grad[~there].isnan().all())
            assert not kept.requires_grad and torch.equal(kept[:, 0], z.float().amax(1))
            # the calls by themselves, in place too
            for p, q in zip(bh.distil_loss(z, idx, u, T, keep=True), (loss, lse, kept)):
                assert same(p, q)
            assert same(bh.distil_loss_backward(dloss, z, idx, u, lse, T, dlogits=z, kept=kept), leaf.grad)


def test_kept_changes_nothing_near_zero():
    for n, v in ROWS:
        z, idx, u = case(n, v, 5, torch.float32, v)
        loss, lse, kept = bh.distil_loss(z, idx, u, keep=True)
        assert bool((lse.abs() < 16).all())
        assert torch.equal(bh.distil_loss_backward(loss, z, idx, u, lse), bh.distil_loss_backward(loss, z, idx, u, lse, kept=kept))


def test_kept_of_rows_that_are_not_finite():
    for v in (40, 3000, 30_000):
        z, idx, u = case(4, v, 5, torch.float32, v)
        z[0], z[1, v // 2], z[2, v // 3] = -math.inf, NAN, math.inf
        leaf = z.clone().requires_grad_()
        loss, lse, kept = bh.distil_loss(leaf, idx, u, keep=True)
        loss.sum().backward()
        assert bool(loss[:3].isnan().all()) and bool(leaf.grad[:3].isnan().any(1).all()) and bool(leaf.grad[3].isfinite().all())
        want = bh.distil_loss_backward(torch.ones(4, device=DEV), z, idx, u, lse)
        assert torch.equal(leaf.grad[3], want[3])


def test_kept_is_refused():
    z, idx, u = case(4, 50, 5, torch.float32, 1)
    loss, lse, kept = bh.distil_loss(z, idx, u, keep=True)
    for bad in (kept[:3], kept.double(), kept.t(), kept.cpu(), lse):
        with pytest.raises(ValueError, match="kept"):
            bh.distil_loss_backward(loss, z, idx, u, lse, kept=bad)
