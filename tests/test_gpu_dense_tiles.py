"""The dense operators at sizes that take each kind of tile, with sums shared out and not, and ends that fall inside a slice.

Tolerances are those of the operators' own tests."""
import pytest
import torch

import paper_2212_11506_amd as bh
from tests.test_gpu_gated import ACTS, U, act64, act_error, check_backward, check_forward, close, mat, operands
from tests.test_gpu_linear8 import check, ints, quantise64
from tests.test_gpu_linear8 import mat as values

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALVES = [torch.float16, torch.bfloat16]


def say(*a):
    print(*a, flush=True)


# tiles of 256: K of one to thirty-three slices, with and without an end inside one, several tiles a block
@pytest.mark.parametrize("dtype,n,d,f", [(t, *c) for t in HALVES for c in [(6464, 72, 727), (5542, 128, 863), (2600, 2056, 2050), (4700, 264, 4300), (2600, 2048, 2050)]]
                         + [(torch.float32, *c) for c in [(2114, 40, 2944), (3275, 64, 1986), (2200, 300, 3001), (697, 35, 2209), (2500, 20, 200)]])
def test_forward(dtype, n, d, f):
    say(f"[tiles] forward {n} x {d} -> {f} {dtype}")
    x, gate, up = mat(n, d, dtype, 1), mat(f, d, dtype, 2, 0, d ** -0.5), mat(f, d, dtype, 3, 0, d ** -0.5)
    for kind in ("silu", "gelu"):
        got = bh.gated_layer(x, gate, up, kind, keep=True)
        check_forward(x, gate, up, kind, *got)
        assert torch.equal(bh.gated_layer(x, gate, up, kind), got[0])


@pytest.mark.parametrize("dtype,n,d,f", [(t, *c) for t in HALVES for c in [
    (66, 2237, 2193), (6619, 395, 2343), (7222, 1323, 30), (7210, 258, 2554), (8546, 66, 2174), (32, 2851, 518), (1715, 1808, 30), (8769, 68, 1476), (6400, 512, 2048)]]
    + [(torch.float32, *c) for c in [(3320, 1729, 886), (4247, 707, 1662), (34, 2273, 2838), (4487, 2776, 32), (8788, 79, 720), (8549, 335, 30), (1507, 197, 2051), (30, 710, 2076)]])
def test_backward(dtype, n, d, f):
    say(f"[tiles] backward {n} x {d} -> {f} {dtype}")
    o = operands(n, d, f, dtype)
    got = bh.gated_layer_backward(*o)
    check_backward(*o, "silu", got)
    for p, q in zip(got, bh.gated_layer_backward(*o)):
        assert torch.equal(p, q)


def test_backward_ends_inside_a_slice():
    """NaN in the last points stays in their own rows of dx; behind the last point nothing is read."""
    for dtype in HALVES + [torch.float32]:
        for n, d, f in ((6621, 392, 2344), (2001, 64, 96), (6619, 395, 2343)):
            say(f"[tiles] last points {n} x {d} -> {f} {dtype}")
            dh, x, gate, up, a, b = operands(n, d, f, dtype)
            wide = torch.full((n + 70, d), float("nan"), dtype=dtype, device=DEV)  # rows behind the last are NaN
            wide[:n] = x
            want = bh.gated_layer_backward(dh, x, gate, up, a, b)
            got = bh.gated_layer_backward(dh, wide[:n], gate, up, a, b)
            assert all(torch.equal(p, q) for p, q in zip(want, got))
            dh = dh.clone()
            dh[n - 1] = float("nan")
            dx = bh.gated_layer_backward(dh, x, gate, up, a, b)[0]
            assert torch.equal(dx[:-1], want[0][:-1]) and bool(dx[-1].isnan().all())


@pytest.mark.parametrize("dtype", HALVES + [torch.float32])
@pytest.mark.parametrize("n,d,f", [(4897, 144, 1905), (7918, 256, 1545), (9000, 2000, 4100), (2913, 16, 1026), (5000, 2000, 2000)])
def test_linear(n, d, f, dtype):
    say(f"[tiles] 8 bits {n} x {d} -> {f} {dtype}")
    w, ws, bias = ints(f, d, 2), values(f, 1, torch.float32, 4).abs().flatten() / d, values(f, 1, dtype, 5).flatten()
    q, s = ints(n, d, 1), values(n, 1, torch.float32, 3).abs().flatten()
    check(q, s, w, ws, bias, bh.linear_i8(q, w, ws, s, bias, dtype=dtype))
    x = values(n, d, dtype, 6)
    out = bh.linear_i8(x, w, ws, bias=bias)
    check(*quantise64(x), w, ws, bias, out)


@pytest.mark.parametrize("kind", HALVES + [torch.float32])
@pytest.mark.parametrize("dtype", HALVES + [torch.float32])
def test_linear_of_one_type_to_another(kind, dtype):
    for n, d, f in ((1, 777, 100), (5, 128, 33), (16, 512, 40), (16, 513, 40), (90, 300, 50)):
        w, ws = ints(f, d, 2, 3), values(f, 1, torch.float32, 4).abs().flatten() / d
        x = values(n, d, kind, 6, 5)
        x[0, d // 2] = 3.0
        out = bh.linear_i8(x, w, ws, dtype=dtype)
        assert out.dtype == dtype
        check(*quantise64(x), w, ws, None, out)


# more than a few points, and few tiles: one block of 64 points, several, an end inside one, and one feature more than is shared
FEW = [(17, 128, 15), (64, 4096, 33), (65, 260, 256), (130, 72, 700), (1000, 144, 250), (1025, 400, 240), (1025, 400, 241), (64, 272, 4097)]


@pytest.mark.parametrize("dtype", HALVES + [torch.float32])
@pytest.mark.parametrize("n,d,f", FEW + [(65, 777, 100), (200, 131, 20)])
def test_forward_of_few_tiles(n, d, f, dtype):
    x, gate, up = mat(n, d, dtype, 1, 8), mat(f, d, dtype, 2, 16, d ** -0.5), mat(f, d, dtype, 3, 0, d ** -0.5)
    for kind in ACTS:
        got = bh.gated_layer(x, gate, up, kind, keep=True)
        check_forward(x, gate, up, kind, *got)
        assert torch.equal(bh.gated_layer(x, gate, up, kind), got[0])
    x = x.clone()
    x[n // 2, d - 1] = float("nan")  # stays in its row
    h = bh.gated_layer(x, gate, up, kind)
    assert bool(h[n // 2].isnan().all()) and torch.equal(h[: n // 2], got[0][: n // 2]) and torch.equal(h[n // 2 + 1 :], got[0][n // 2 + 1 :])


@pytest.mark.parametrize("dtype", HALVES + [torch.float32])
@pytest.mark.parametrize("n,d,f", FEW)
def test_linear_of_few_tiles(n, d, f, dtype):
    w, ws, bias = ints(f, d, 2), values(f, 1, torch.float32, 4).abs().flatten() / d, values(f, 1, dtype, 5).flatten()
    q, s = ints(n, d, 1), values(n, 1, torch.float32, 3).abs().flatten()
    check(q, s, w, ws, bias, bh.linear_i8(q, w, ws, s, bias, dtype=dtype))
    x = values(n, d, dtype, 6)
    check(*quantise64(x), w, ws, bias, bh.linear_i8(x, w, ws, bias=bias))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("n,d,f", [(2000, 10, 40), (3000, 1, 2), (20, 200, 300), (1, 2000, 700), (63, 65, 2000), (20_000, 50, 80)])
def test_backward_of_few_outputs(n, d, f, dtype):
    """Sums of few outputs are formed from gradients of 32 bits: nothing but the outputs is rounded to the type."""
    o = operands(n, d, f, dtype)
    for kind in ACTS:
        got = bh.gated_layer_backward(*o, kind)
        dh, x, gate, up, a, b = (t.double() for t in o)
        value, slope, size = act64(a, kind)
        rel = act_error(a, kind, dtype) + 4 * U
        da, db = dh * b * slope, dh * value
        ta, tb = rel * (dh * b).abs() * size, rel * db.abs()
        k = (2 * f + 8) * U
        close(got[0], da @ gate + db @ up, ta @ gate.abs() + tb @ up.abs() + k * (da.abs() @ gate.abs() + db.abs() @ up.abs()), dtype)
        k = (n + 8) * U
        for grad, e, t in ((got[1], da, ta), (got[2], db, tb)):
            e, t = e.T.contiguous(), t.T.contiguous()
            close(grad, e @ x, t @ x.abs() + k * (e.abs() @ x.abs()), dtype)
