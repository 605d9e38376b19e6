"""Rows of a hundred thousand features and more: the sums of a row do not gather rounding errors.

A sum of d equal values in fp64 is exact up to d = 2^29, so a constant row's mean is its value, its output the bias, its
variance zero.  Else a sum's error is 2^-53 d of its terms' magnitude, far below one fp32 rounding: statistics are within
2^-23 of their size, outputs within a few of these and their own rounding."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
EPS = 1e-5
WIDTHS = [16_385, 100_000, 1 << 20, (1 << 20) + 3]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", WIDTHS)
def test_constant_rows(d, dtype):
    x = torch.full((2, d), 100.3, dtype=dtype, device=DEV)
    b = torch.linspace(-1, 1, d, device=DEV)
    y, mean, rstd = bh.layer_norm(x, None, b, eps=EPS)
    print(f"[norm] d={d} {dtype} mean {float(mean[0])} rstd {float(rstd[0])} y {float((y.float() - b.to(dtype).float()).abs().max())}",
          flush=True)
    assert bool((mean == x[:, 0].float()).all())
    assert bool(((rstd.double() - EPS ** -0.5).abs() <= 8 * U * EPS ** -0.5).all())
    assert torch.equal(y, b.to(dtype).expand(2, d))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", WIDTHS)
def test_little_spread_over_a_large_offset(d, dtype):
    g = torch.Generator().manual_seed(d)
    x = (100.3 + 0.5 * torch.randn(3, d, generator=g)).to(dtype)
    w, b = 1.0 + 0.2 * torch.randn(d, generator=g), 0.1 * torch.randn(d, generator=g)
    y, mean, rstd = (t.double().cpu() for t in bh.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV), eps=EPS))
    X = x.double()
    m = X.mean(1)
    r = ((X - m[:, None]).square().mean(1) + EPS) ** -0.5
    assert bool(((mean - m).abs() <= 2 * U * m.abs()).all())
    # the mean's rounding enters the squares by its own square only
    assert bool(((rstd - r).abs() <= 8 * U * r).all())
    want = (X - m[:, None]) * r[:, None] * w.double() + b.double()
    tol = w.double().abs() * ((2 * U * m.abs() * r)[:, None] + 16 * U * ((X - m[:, None]) * r[:, None]).abs()) + 4 * U * want.abs()
    tol = tol + 4 * U * b.double().abs() + HALF[dtype] * (want.abs() + tol) + TINY[dtype]
    assert bool(((y - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward_of_one_sided_gradients(d, dtype):
    """dy that is nearly the same everywhere: g - mean(g) leaves what differs, not what a long sum has lost."""
    g = torch.Generator().manual_seed(d + 1)
    x = (3.0 + torch.randn(2, d, generator=g)).to(dtype)
    dy = torch.full((2, d), 0.1).to(dtype)
    X, D = x.double(), dy.double()
    m = X.mean(1)
    r = ((X - m[:, None]).square().mean(1) + EPS) ** -0.5
    mean, rstd = m.float(), r.float()
    dx, dw, db = bh.layer_norm_backward(dy.to(DEV), x.to(DEV), None, mean.to(DEV), rstd.to(DEV))
    m, r = mean.double()[:, None], rstd.double()[:, None]
    xh = (X - m) * r
    want = r * (D - D.mean(1, keepdim=True) - xh * (D * xh).mean(1, keepdim=True))
    # a few roundings of g and of xh s2, each of its own size
    tol = 4 * U * r * (D.abs() + xh.abs() * (D * xh).abs().mean(1, keepdim=True))
    tol = tol + HALF[dtype] * (want.abs() + tol)
    err = (dx.double().cpu() - want).abs()
    print(f"[norm] backward d={d} {dtype} {float((err / tol).max()):.2f} of the bound", flush=True)
    assert bool((err <= tol).all())
    for got, exact in ((dw, (D * xh).sum(0)), (db, D.sum(0))):
        size = (D * xh).abs().sum(0) if got is dw else D.sum(0)
        assert bool(((got.double().cpu() - exact).abs() <= 8 * U * size + HALF[dtype] * (exact.abs() + 8 * U * size)).all())
