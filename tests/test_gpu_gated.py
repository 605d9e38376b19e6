"""The gated layer, forward and backward, against the formulas in 64 bits and against differences.

Tolerances: u = 2^-24 is half a unit in the last place of fp32.  A sum of k terms in any order is within k u of the sum of
magnitudes.  The activations: silu's exponential takes an argument off by |a| u, its instructions are off by units in the last
place; gelu's erfc takes one off by u, which it multiplies by a^2 far below zero; (a^2 + |a| + 16) 2u of the value covers
both.  For 16-bit types gelu's tail is a fit of degree 5 that is off by 1.8e-5 of its value at most; the tail enters the value
and the slope as a part of their size or less, so 2e-5 more of them covers it and its roundings.  An operand or an output of t bits is rounded by half a unit in its last place."""
import numpy as np
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}  # half the spacing of subnormals
TYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = ["silu", "gelu"]


def say(*a):
    print(*a, flush=True)


def mat(n, d, dtype, seed, pad=0, scale=1.0):
    """n x d values, the first columns of rows d + pad long: what lies behind is NaN."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((n, d + pad), float("nan"), dtype=dtype)
    buf[:, :d] = (scale * torch.randn(n, d, generator=g)).to(dtype)
    return buf.to(DEV)[:, :d]


def act64(a, kind):
    """Value, slope, and the slope's terms without their signs."""
    if kind == "silu":
        s = torch.sigmoid(a)
        return a * s, s * (1 + a * (1 - s)), s * (1 + a.abs() * (1 - s))
    phi = 0.5 * torch.special.erfc(a * -np.sqrt(0.5))  # exact far below zero too
    pdf = torch.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    return a * phi, phi + a * pdf, phi + a.abs() * pdf


def act_error(a, kind, dtype):
    """How far an activation's value or slope may be off, relative to its size."""
    return (a * a + a.abs() + 16) * 2 * U + (2e-5 if kind == "gelu" and dtype != torch.float32 else 0.0)


def close(got, want, tol, dtype):
    tol = tol + HALF[dtype] * (want.abs() + tol) + TINY[dtype]
    err = (got.double() - want).abs()
    assert got.dtype == dtype and bool((err <= tol).all()), float((err / tol).max())


def check_forward(x, gate, up, kind, h, a, b):
    x64, g64, u64 = x.double(), gate.double(), up.double()
    k = (x.shape[1] + 4) * U
    ea, eb = x64 @ g64.T.contiguous(), x64 @ u64.T.contiguous()
    ta, tb = k * (x64.abs() @ g64.abs().T.contiguous()), k * (x64.abs() @ u64.abs().T.contiguous())
    value = act64(ea, kind)[0]
    tol = 1.13 * ta * (eb.abs() + tb) + value.abs() * tb + act_error(ea, kind, x.dtype) * (value * eb).abs()
    close(h, value * eb, tol, x.dtype)
    if a is not None:
        close(a, ea, ta, x.dtype)
        close(b, eb, tb, x.dtype)


# widths off every tile and vector, single rows and features, several slices of K
SIZES = [(1, 1, 1), (1, 512, 256), (3, 2, 5), (16, 64, 33), (17, 50, 200), (63, 77, 64), (64, 64, 64), (65, 129, 130), (130, 333, 31),
         (300, 8, 100), (257, 1000, 48), (1000, 96, 17), (5, 2053, 70)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,f", SIZES)
def test_forward(n, d, f, dtype):
    for kind in ACTS:
        for pad in (0, 3, 8):
            say(f"[gated] forward {n} x {d} -> {f} pad {pad} {kind} {dtype}")
            x, gate, up = mat(n, d, dtype, 1, pad), mat(f, d, dtype, 2, pad, d ** -0.5), mat(f, d, dtype, 3, 0, d ** -0.5)
            h, a, b = bh.gated_layer(x, gate, up, kind, keep=True)
            check_forward(x, gate, up, kind, h, a, b)
            assert torch.equal(bh.gated_layer(x, gate, up, kind), h)


# enough tiles for the larger kinds of blocks
LARGE = [(4099, 200, 2056), (4099, 203, 2051), (2000, 64, 1024), (2001, 72, 1000), (70_001, 50, 200), (20_000, 24, 100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,f", LARGE)
def test_forward_large(n, d, f, dtype):
    say(f"[gated] forward {n} x {d} -> {f} {dtype}")
    x, gate, up = mat(n, d, dtype, 1), mat(f, d, dtype, 2, 0, d ** -0.5), mat(f, d, dtype, 3, 0, d ** -0.5)
    check_forward(x, gate, up, "silu", *bh.gated_layer(x, gate, up, keep=True))


def test_activations_over_their_range():
    """One feature, weights of 1: a and b are x itself."""
    x = torch.cat([torch.linspace(-40, 40, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, -100.0, 100.0, -1e4, 1e4, 3e18, -3e18])]).to(DEV)[:, None]
    one = torch.ones(1, 1, device=DEV)
    for kind in ACTS:
        h = bh.gated_layer(x.contiguous(), one, one, kind)
        x64 = x.double()
        value = act64(x64, kind)[0]
        close(h, value * x64, (x64 * x64 + x64.abs() + 16).clamp(max=1e4) * 2 * U * (value * x64).abs() + 2.0 ** -126, torch.float32)
    for t in (torch.float16, torch.bfloat16):
        z = torch.linspace(-20, 20, 501).to(t).to(DEV)[:, None]
        for kind in ACTS:
            z64 = z.double()
            value = act64(z64, kind)[0]
            close(bh.gated_layer(z, one.to(t), one.to(t), kind), value * z64,
                  act_error(z64, kind, t) * (value * z64).abs() + 2.0 ** -126, t)


def check_backward(dh, x, gate, up, a, b, kind, got):
    dtype = x.dtype
    dh64, x64, g64, u64, a64, b64 = (t.double() for t in (dh, x, gate, up, a, b))
    value, slope, size = act64(a64, kind)
    rel = act_error(a64, kind, dtype)
    da, db = dh64 * b64 * slope, dh64 * value
    ta = rel * (dh64 * b64).abs() * size
    tb = rel * db.abs()
    ta, tb = (t + HALF[dtype] * (e.abs() + t) + TINY[dtype] for t, e in ((ta, da), (tb, db)))
    f, n = gate.shape[0], x.shape[0]
    ag, au, ax = g64.abs(), u64.abs(), x64.abs()
    k = (2 * f + 8) * U
    close(got[0], da @ g64 + db @ u64, ta @ ag + tb @ au + k * (da.abs() @ ag + db.abs() @ au), dtype)
    k = (n + 8) * U
    for grad, e, t in ((got[1], da, ta), (got[2], db, tb)):
        e, t = e.T.contiguous(), t.T.contiguous()
        close(grad, e @ x64, t @ ax + k * (e.abs() @ ax), dtype)


def operands(n, d, f, dtype, pad=0):
    x, gate, up = mat(n, d, dtype, 1, pad), mat(f, d, dtype, 2, pad, d ** -0.5), mat(f, d, dtype, 3, 0, d ** -0.5)
    return mat(n, f, dtype, 4, pad, 0.1), x, gate, up, mat(n, f, dtype, 5, pad), mat(n, f, dtype, 6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,f", SIZES)
def test_backward(n, d, f, dtype):
    for kind in ACTS:
        for pad in (0, 3):
            say(f"[gated] backward {n} x {d} -> {f} pad {pad} {kind} {dtype}")
            o = operands(n, d, f, dtype, pad)
            got = bh.gated_layer_backward(*o, kind)
            check_backward(*o, kind, got)
            for p, q in zip(got, bh.gated_layer_backward(*o, kind)):
                assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,f", [(4099, 200, 1031), (20_001, 50, 200), (3000, 520, 2000), (30_000, 16, 40)])
def test_backward_large(n, d, f, dtype):
    say(f"[gated] backward {n} x {d} -> {f} {dtype}")
    o = operands(n, d, f, dtype)
    check_backward(*o, "silu", bh.gated_layer_backward(*o))


def test_gradient_against_differences():
    n, d, f = 7, 9, 11
    for kind in ACTS:
        x, gate, up = (mat(*s, torch.float32, k).requires_grad_() for k, s in enumerate([(n, d), (f, d), (f, d)]))
        r = mat(n, f, torch.float32, 9)
        (bh.gated_layer(x, gate, up, kind) * r).sum().backward()

        def loss(ts):
            a, b = ts[0] @ ts[1].T.contiguous(), ts[0] @ ts[2].T.contiguous()
            return float((act64(a, kind)[0] * b * r.double()).sum())
        base = [t.detach().double() for t in (x, gate, up)]
        for which, t in enumerate((x, gate, up)):
            for at in range(0, t.numel(), 5):
                step = 1e-5
                ends = []
                for sign in (1, -1):
                    moved = [q.clone() for q in base]
                    moved[which].view(-1)[at] += sign * step
                    ends.append(loss(moved))
                # central differences: step^2 of the third derivative; the gradient's own sums of at most 77 terms
                assert abs((ends[0] - ends[1]) / (2 * step) - float(t.grad.view(-1)[at])) <= 2e-5 * (1 + float(t.grad.abs().max()))


def test_no_points():
    for t in TYPES:
        x, gate, up = mat(0, 5, t, 1), mat(7, 5, t, 2), mat(7, 5, t, 3)
        h, a, b = bh.gated_layer(x, gate, up, keep=True)
        assert h.shape == a.shape == b.shape == (0, 7)
        dx, dgate, dup = bh.gated_layer_backward(h, x, gate, up, a, b)
        assert dx.shape == (0, 5) and not dgate.any() and not dup.any() and dgate.shape == dup.shape == (7, 5)


def test_nan_and_infinity_stay_in_their_rows():
    """A point's NaN or infinity does not reach the others, nor the values behind a row's end."""
    for t in TYPES:
        for n, d, f in ((70, 40, 48), (70, 43, 45), (300, 136, 64)):
            x, gate, up = mat(n, d, t, 1, 5), mat(f, d, t, 2, 3), mat(f, d, t, 3)
            want = bh.gated_layer(x, gate, up)
            y = x.clone()
            y[3, 1], y[n - 1, d - 1] = float("nan"), float("inf")
            got = bh.gated_layer(y, gate, up)
            rows = [r for r in range(n) if r not in (3, n - 1)]
            assert torch.equal(got[rows], want[rows]) and bool(got[3].isnan().all()) and not bool(got[n - 1].isfinite().any())


def test_rows_between_others_are_left_alone():
    """Outputs with gaps between rows and at odd alignments: nothing else is written."""
    for t in TYPES:
        for off, gap in ((0, 0), (1, 0), (3, 5), (8, 8)):
            n, d, f = 131, 40, 77
            x, gate, up = mat(n, d, t, 1), mat(f, d, t, 2), mat(f, d, t, 3)
            buf = torch.full((n * (f + gap) + off + 8,), 7.0, dtype=t, device=DEV)
            out = buf[off:off + n * (f + gap)].view(n, f + gap)[:, :f]
            assert bh.gated_layer(x, gate, up, out=out) is out
            assert torch.equal(out, bh.gated_layer(x, gate, up))
            rest = buf.clone()
            rest[off:off + n * (f + gap)].view(n, f + gap)[:, :f] = 7.0
            assert bool((rest == 7.0).all())


def test_one_row_for_all():
    for t in TYPES:
        n, d, f = 40, 33, 20
        x, gate, up = mat(1, d, t, 1).expand(n, d), mat(f, d, t, 2), mat(f, d, t, 3)
        h, a, b = bh.gated_layer(x, gate, up, keep=True)
        assert torch.equal(h, bh.gated_layer(x.contiguous(), gate, up))
        dh = mat(1, f, t, 4).expand(n, f)
        for p, q in zip(bh.gated_layer_backward(dh, x, gate, up, a, b),
                        bh.gated_layer_backward(dh.contiguous(), x.contiguous(), gate, up, a, b)):
            assert torch.equal(p, q)


def test_in_torch_graph():
    n, d, f = 50, 24, 30
    for kind in ACTS:
        x, gate, up = (mat(*s, torch.float32, k).requires_grad_() for k, s in enumerate([(n, d), (f, d), (f, d)]))
        h, a, b = bh.gated_layer(x, gate, up, kind, keep=True)
        assert h.requires_grad and not a.requires_grad and not b.requires_grad
        r = mat(n, f, torch.float32, 8)
        h.backward(r)
        for got, want in zip((x.grad, gate.grad, up.grad), bh.gated_layer_backward(r, *(t.detach() for t in (x, gate, up)), a, b, kind)):
            assert torch.equal(got, want)
        grads = [x.grad.clone(), gate.grad.clone(), up.grad.clone()]
        # only what is wanted; a gradient that is one value for all
        x.grad = gate.grad = up.grad = None
        bh.gated_layer(x.detach(), gate, up.detach(), kind).sum().backward()
        assert x.grad is None and up.grad is None
        g0 = gate.grad.clone()
        gate.grad = None
        bh.gated_layer(x, gate, up, kind).sum().backward()
        assert torch.equal(gate.grad, g0)
        # weights that two layers share: their gradients add up
        x.grad = gate.grad = up.grad = None
        (bh.gated_layer(x, gate, up, kind) * r).sum().add((bh.gated_layer(x, gate, up, kind) * r).sum()).backward()
        for got, want in zip((x.grad, gate.grad, up.grad), grads):
            assert torch.equal(got, want + want)
        with pytest.raises(ValueError, match="gradient"):
            bh.gated_layer(x, gate, up, kind, out=torch.empty(n, f, device=DEV))
        y = bh.gated_layer(x, gate, up, kind)
        g, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()


@pytest.mark.parametrize("n,d,f", [(300, 50, 200), (3, 64, 33), (300, 300, 512), (1000, 144, 250), (2600, 512, 2304)])
def test_one_of_the_products_kept(n, d, f):
    """The C call may leave out a or b: the others are written as with both."""
    lib, t, stream = bh.load_library(), torch.float16, torch.cuda.current_stream().cuda_stream
    x, gate, up = mat(n, d, t, 1), mat(f, d, t, 2, 0, d ** -0.5), mat(f, d, t, 3, 0, d ** -0.5)
    want = bh.gated_layer(x, gate, up, "gelu", keep=True)
    for which in (1, 2):
        got = [torch.full((n, f), -7.0, dtype=t, device=DEV) for _ in range(3)]
        a, b = (got[1].data_ptr(), None) if which == 1 else (None, got[2].data_ptr())
        assert lib.bhtsne_gated_layer(x.data_ptr(), d, gate.data_ptr(), d, up.data_ptr(), d, n, d, f, 1, 1, got[0].data_ptr(), f, a, f, b, f, stream) == 0
        torch.cuda.synchronize()
        check_forward(x, gate, up, "gelu", got[0], got[1] if which == 1 else want[1], got[2] if which == 2 else want[2])
        assert bool((got[3 - which] == -7.0).all())
