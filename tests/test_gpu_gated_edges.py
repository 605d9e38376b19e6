"""The gated layer where its values leave the finite numbers."""
import math

import pytest
import torch

import paper_2212_11506_amd as bh
from tests.test_gpu_gated import ACTS, TYPES, mat, operands

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = math.inf


# a few points, few tiles, short rows, tiles of each size, rows off 16 bytes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,f", [(4, 40, 48), (4, 1, 1), (40, 8, 40), (70, 136, 64), (70, 43, 45), (300, 200, 1000), (2600, 512, 2304), (2001, 131, 1000)])
def test_infinite_products(n, d, f, dtype):
    """act(a) of an infinite a: infinity above zero, NaN below, by either activation; only in its own place."""
    x, gate, up = mat(n, d, dtype, 1).abs() + 1, mat(f, d, dtype, 2).abs() + 0.5, mat(f, d, dtype, 3).abs() + 0.5
    gate[1::2] *= -1  # a below zero
    r = n // 2
    for kind in ACTS:
        want = bh.gated_layer(x, gate, up, kind, keep=True)
        y = x.clone()
        y[r, d - 1] = INF
        h, a, b = bh.gated_layer(y, gate, up, kind, keep=True)
        assert bool((a[r, 0::2] == INF).all()) and bool((a[r, 1::2] == -INF).all()) and bool((b[r] == INF).all())
        assert bool((h[r, 0::2] == INF).all()) and bool(h[r, 1::2].isnan().all())
        for p, q in zip((h, a, b), want):
            assert torch.equal(p[:r], q[:r]) and torch.equal(p[r + 1:], q[r + 1:])
        assert torch.equal(bh.gated_layer(y, gate, up, kind).nan_to_num(nan=-7.0), h.nan_to_num(nan=-7.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_that_overflow(dtype):
    """a beyond the largest number beside a finite b."""
    for n in (4, 40, 900):
        x = torch.full((n, 8), 3e37, dtype=dtype, device=DEV)
        gate, up = torch.full((40, 8), 2.0, dtype=dtype, device=DEV), torch.full((40, 8), 2.0 ** -120, dtype=dtype, device=DEV)
        for kind in ACTS:
            assert bool((bh.gated_layer(x, gate, up, kind) == INF).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,f", [(20, 30, 40), (900, 136, 320), (901, 131, 333), (6400, 512, 2048)])
def test_backward_of_infinite_products(n, d, f, dtype):
    """dup is a sum of dh act(a) x: infinite where a is, by either activation; other features and points are as without."""
    dh, x, gate, up, a, b = operands(n, d, f, dtype)
    x, up, dh = x.abs() + 0.5, up.abs() + 0.5, dh.abs() + 0.125
    r, j = n // 3, f // 2
    for kind in ACTS:
        want = bh.gated_layer_backward(dh, x, gate, up, a, b, kind)
        wild = a.clone()
        wild[r, j] = INF
        dx, dgate, dup = bh.gated_layer_backward(dh, x, gate, up, wild, b, kind)
        assert bool((dup[j] == INF).all()) and bool(dgate[j].isnan().all()) and not bool(dx[r].isfinite().any())
        for p, q, at in ((dx, want[0], r), (dgate, want[1], j), (dup, want[2], j)):
            assert torch.equal(p[:at], q[:at]) and torch.equal(p[at + 1:], q[at + 1:])
