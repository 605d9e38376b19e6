"""Layer norm, forward and backward, against the formulas in 64 bits and against differences.

Tolerances: u = 2^-24 is half a unit in the last place of fp32.  A sum whose longest chain of additions has k
terms is within k u of the sum of magnitudes; a row's chain is at most its values per lane (16, or d / 1024 in a
long row), 6 exchanges in the wave and 16 waves, so `terms` below bounds it with room for the few other
operations.  An output of t bits is rounded once, by half a unit in its last place."""
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
EPS = 1e-5


def say(*a):
    print(*a, flush=True)


def terms(d):
    return 64.0 + d / 1024


def rows(n, d, dtype, seed, pad=0, scale=1.0, offset=0.3):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((n, d + pad), float("nan"), dtype=dtype)
    buf[:, :d] = (scale * torch.randn(n, d, generator=g) + offset).to(dtype)
    return buf.to(DEV)[:, :d]


def vec(d, dtype, seed, mean, spread):
    g = torch.Generator().manual_seed(seed)
    return (mean + spread * torch.randn(d, generator=g)).to(dtype).to(DEV)


def forward64(x, w, b, eps):
    x = x.double().cpu()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None]
    if w is not None:
        y = y * w.double().cpu()
    return (y if b is None else y + b.double().cpu()), mean, rstd


def check_forward(x, w, b, got, eps=EPS):
    y, mean, rstd = got
    ye, me, re = forward64(x, w, b, eps)
    d = x.shape[1]
    k = terms(d) * U
    big = x.double().cpu().abs().amax(1)
    assert mean.dtype == rstd.dtype == torch.float32 and y.dtype == x.dtype and y.shape == x.shape
    assert bool(((mean.double().cpu() - me).abs() <= k * big + 1e-45).all())
    # the centred squares: 2 k of the values' size against their spread
    spread = 1.0 / re
    assert bool(((rstd.double().cpu() - re).abs() <= re * (k + 2 * k * big / spread)).all())
    wa = 1.0 if w is None else w.double().cpu().abs()
    ba = 0.0 if b is None else b.double().cpu().abs()
    xh = forward64(x, None, None, eps)[0].abs()
    tol = wa * (k * (big * re)[:, None] + xh * (k + 2 * k * big / spread)[:, None]) + 2 * U * (ye.abs() + ba)
    err = (y.double().cpu() - ye).abs()
    tol = tol + HALF[x.dtype] * (ye.abs() + tol) + TINY[x.dtype]
    assert bool((err <= tol).all()), float((err / tol).max())


# widths: one lane's vector, a team of each size, ends inside a vector, a whole block, longer than a block's registers
WIDTHS = [1, 2, 3, 7, 8, 20, 50, 63, 64, 65, 100, 128, 255, 256, 333, 500, 512, 513, 777, 1000, 1024, 1025, 1536, 2048, 4099,
          8192, 16384, 16385, 20000]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_forward(d, dtype):
    for n, pad in ((1, 0), (5, 0), (67, 3), (67, 8)):
        say(f"[norm] forward n={n} d={d} pad={pad} {dtype}")
        x = rows(n, d, dtype, d + n, pad)
        for w, b in ((vec(d, dtype, 1, 1.0, 0.2), vec(d, dtype, 2, 0.0, 0.1)), (vec(d, torch.float32, 3, 1.0, 0.2), None),
                     (None, None)):
            check_forward(x, w, b, bh.layer_norm(x, w, b, eps=EPS))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d", [(2000, 128), (70_001, 50), (30_011, 333), (5000, 2048), (300_007, 3)])
def test_forward_many_rows(n, d, dtype):
    say(f"[norm] forward n={n} d={d} {dtype}")
    x = rows(n, d, dtype, 7)
    w, b = vec(d, dtype, 1, 1.0, 0.2), vec(d, dtype, 2, 0.0, 0.1)
    check_forward(x, w, b, bh.layer_norm(x, w, b, eps=EPS))


def back64(dy, x, w, mean, rstd):
    dy, x = dy.double().cpu(), x.double().cpu()
    mean, rstd = mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
    xh = (x - mean) * rstd
    g = dy if w is None else dy * w.double().cpu()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), xh, g


def check_backward(dy, x, w, mean, rstd, got):
    dx, dw, db = got
    n, d = x.shape
    e_dx, e_dw, e_db, xh, g = back64(dy, x, w, mean, rstd)
    k = terms(d) * U
    ptype = x.dtype if w is None else w.dtype
    assert dx.dtype == x.dtype and dw.dtype == db.dtype == ptype
    r = rstd.double().cpu().abs()[:, None]
    tol = k * r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    err = (dx.double().cpu() - e_dx).abs()
    tol = tol + HALF[x.dtype] * (e_dx.abs() + tol) + TINY[x.dtype]
    assert bool((err <= tol).all()), float((err / tol).max())
    kn = (64.0 + n / 256) * U  # a lane adds up every 1024th row or fewer, a block at most 256 lanes
    dya = dy.double().cpu().abs()
    for out, want, size in ((dw, e_dw, (dya * xh.abs()).sum(0)), (db, e_db, dya.sum(0))):
        err = (out.double().cpu() - want).abs()
        tol = kn * size
        tol = tol + HALF[ptype] * (want.abs() + tol) + TINY[ptype]
        assert bool((err <= tol).all()), float((err / tol).max())


def stats(x, eps=EPS):
    _, mean, rstd = forward64(x, None, None, eps)
    return mean.float().to(DEV), rstd.float().to(DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_backward(d, dtype):
    for n, pad in ((1, 0), (5, 0), (67, 3), (67, 8)):
        say(f"[norm] backward n={n} d={d} pad={pad} {dtype}")
        x, dy = rows(n, d, dtype, d + n, pad), rows(n, d, dtype, d + n + 1, pad, 0.1, 0.01)
        mean, rstd = stats(x)
        for w in (vec(d, dtype, 1, 1.0, 0.2), vec(d, torch.float32, 3, 1.0, 0.2), None):
            check_backward(dy, x, w, mean, rstd, bh.layer_norm_backward(dy, x, w, mean, rstd))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d", [(2000, 128), (70_001, 50), (30_011, 333), (5000, 2048), (300_007, 3), (3000, 16_390)])
def test_backward_many_rows(n, d, dtype):
    say(f"[norm] backward n={n} d={d} {dtype}")
    x, dy = rows(n, d, dtype, 7), rows(n, d, dtype, 8, 0, 0.1, 0.01)
    mean, rstd = stats(x)
    w = vec(d, torch.float32, 1, 1.0, 0.2)
    check_backward(dy, x, w, mean, rstd, bh.layer_norm_backward(dy, x, w, mean, rstd))


def test_backward_against_differences():
    """The loss sum(y r) of the forward pass in 64 bits, moved along random directions, against the gradients."""
    n, d, h = 9, 37, 1e-6
    x, w, b = rows(n, d, torch.float32, 1), vec(d, torch.float32, 2, 1.0, 0.2), vec(d, torch.float32, 3, 0.0, 0.1)
    r = rows(n, d, torch.float32, 4)
    _, mean, rstd = bh.layer_norm(x, w, b, eps=EPS)
    dx, dw, db = bh.layer_norm_backward(r, x, w, mean, rstd)
    loss = lambda x, w, b: float((forward64(x, w, b, EPS)[0] * r.double().cpu()).sum())  # noqa: E731
    at = [t.double().cpu() for t in (x, w, b)]
    for k, grad in enumerate((dx, dw, db)):
        g = torch.Generator().manual_seed(10 + k)
        v = torch.randn(at[k].shape, generator=g, dtype=torch.float64)
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + h * v, at[k] - h * v
        want = (loss(*up) - loss(*down)) / (2 * h)
        got = float((grad.double().cpu() * v).sum())
        # differences: h^2 and 1e-16 / h; the gradient: fp32
        assert abs(got - want) <= 1e-5 * float((grad.double().cpu() * v).abs().sum())


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_broadcast_rows(dtype):
    n, d = 131, 96
    x, w, b = rows(n, d, dtype, 1), vec(d, dtype, 2, 1.0, 0.2), vec(d, dtype, 3, 0.0, 0.1)
    y, mean, rstd = bh.layer_norm(x, w, b)
    dy = rows(n, d, dtype, 4)
    back = bh.layer_norm_backward(dy, x, w, mean, rstd)
    for target in (dy.clone(), None):
        xx = x.clone()
        into = target if target is not None else xx
        again = bh.layer_norm_backward(into if target is not None else dy, xx, w, mean, rstd, dx=into)
        assert again[0].data_ptr() == into.data_ptr()
        assert all(torch.equal(p, q) for p, q in zip(again, back))
    z = x.clone()
    assert torch.equal(bh.layer_norm(z, w, b, out=z)[0], y) and torch.equal(z, y)
    one = dy[:1].expand(n, d)  # the gradient of a sum over points
    assert one.stride(0) == 0
    assert all(torch.equal(p, q) for p, q in zip(bh.layer_norm_backward(one, x, w, mean, rstd),
                                                 bh.layer_norm_backward(one.contiguous(), x, w, mean, rstd)))
    same = x[:1].expand(n, d)
    assert torch.equal(bh.layer_norm(same, w, b)[0], bh.layer_norm(same.contiguous(), w, b)[0])


@pytest.mark.parametrize("d", [16, 700, 16_400])
def test_padding_is_never_written_and_rows_stay_apart(d):
    """Strided outputs leave what lies between rows; a row of NaN or infinities spoils that row alone, and the
    weights' gradients as the sums say."""
    n = 33
    x = rows(n, d, torch.bfloat16, 1)
    x = x.clone()
    x[3] = float("nan")
    x[7, d // 2] = float("inf")
    out = torch.full((n, d + 5), 42.0, dtype=torch.bfloat16, device=DEV)
    y, mean, rstd = bh.layer_norm(x, out=out[:, :d])
    assert bool((out[:, d:] == 42.0).all())
    fine = [i for i in range(n) if i not in (3, 7)]
    assert bool(torch.isfinite(y[fine]).all()) and bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[7]).all())
    assert bool(torch.isnan(mean[3])) and bool(torch.isinf(mean[7]))
    check_forward(x[fine].contiguous(), None, None, tuple(t[fine] for t in (y, mean, rstd)))
    dy = rows(n, d, torch.bfloat16, 2)
    dx, dw, db = bh.layer_norm_backward(dy, x, None, mean, rstd)
    assert bool(torch.isfinite(dx[fine]).all()) and bool(torch.isnan(dx[3]).all())
    assert bool(torch.isnan(dw).all()) and bool(torch.isfinite(db).all())


def test_constant_rows_and_far_offsets():
    """A row without spread has rstd = eps^(-1/2) and gives the bias; a spread far below the offset survives."""
    x = torch.full((4, 300), 3.25, device=DEV)
    b = vec(300, torch.float32, 1, 0.0, 1.0)
    y, mean, rstd = bh.layer_norm(x, None, b, eps=1e-4)
    assert torch.equal(y, b.expand(4, 300)) and bool((mean == 3.25).all())
    assert bool(((rstd - 100.0).abs() <= 100.0 * 8 * U).all())
    x = rows(16, 500, torch.float32, 2, 0, 1.0, 1000.0)
    check_forward(x, None, None, bh.layer_norm(x))
    one = rows(9, 1, torch.float32, 3)
    assert bool((bh.layer_norm(one)[0] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [6, 64, 300, 9000])
def test_starts_off_every_alignment(d, dtype):
    """Rows, weights and outputs that begin one element behind an aligned address give what aligned ones give."""
    n = 41
    x, dy, w, b = rows(n, d, dtype, 1), rows(n, d, dtype, 2), vec(d, dtype, 3, 1.0, 0.2), vec(d, dtype, 4, 0.0, 0.1)
    shift = lambda t: torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(t.shape)  # noqa: E731
    got = bh.layer_norm(shift(x), shift(w), shift(b), out=shift(torch.zeros_like(x)))
    check_forward(x, w, b, got)
    back = bh.layer_norm_backward(shift(dy), shift(x), shift(w), shift(got[1]), shift(got[2]), dx=shift(torch.zeros_like(x)))
    check_backward(dy, x, w, got[1], got[2], back)


@pytest.mark.parametrize("ptype", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 50, 96, 504, 1000, 2000])
def test_parameters_off_every_alignment(d, dtype, ptype):
    """Weights and biases that start anywhere give what aligned copies of them give, alone and together."""
    if ptype != dtype and ptype != torch.float32:
        return  # parameters are fp32 or of x's type
    x, dy = rows(37, d, dtype, 1), rows(37, d, dtype, 2, 0, 0.1, 0.01)
    w, b = vec(d + 8, ptype, 3, 1.0, 0.2), vec(d + 8, ptype, 4, 0.0, 0.1)
    for i, j in ((1, 1), (2, 3), (4, 2), (7, 0), (0, 5)):
        wi, bj = w[i:i + d], b[j:j + d]
        wc, bc = wi.clone(), bj.clone()
        for ww, bb, wa, ba in ((wi, bj, wc, bc), (wi, None, wc, None), (None, bj, None, bc)):
            got, want = bh.layer_norm(x, ww, bb), bh.layer_norm(x, wa, ba)
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        check_forward(x, wi, bj, bh.layer_norm(x, wi, bj, eps=EPS))
        mean, rstd = want[1:]
        assert all(torch.equal(p, q) for p, q in zip(bh.layer_norm_backward(dy, x, wi, mean, rstd),
                                                     bh.layer_norm_backward(dy, x, wc, mean, rstd)))


def test_arrays_beyond_the_caches():
    """Rows of a 280 MB array, which are read and written past the caches, come out as they do in parts."""
    n, d = 550_000, 256
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((n, d), generator=g, device=DEV).to(torch.bfloat16)
    dy = (0.1 * torch.randn((n, d), generator=g, device=DEV) + 0.01).to(torch.bfloat16)
    w, b = vec(d, torch.float32, 2, 1.0, 0.2), vec(d, torch.float32, 3, 0.0, 0.1)
    assert x.numel() * 2 > 256 << 20
    y, mean, rstd = bh.layer_norm(x, w, b)
    dx, dw, db = bh.layer_norm_backward(dy, x, w, mean, rstd)
    half, sums = n // 2 + 3, 0.0
    for i, j in ((0, half), (half, n)):
        part = bh.layer_norm(x[i:j], w, b)
        assert all(torch.equal(p, q[i:j]) for p, q in zip(part, (y, mean, rstd)))
        back = bh.layer_norm_backward(dy[i:j], x[i:j], w, mean[i:j], rstd[i:j])
        assert torch.equal(back[0], dx[i:j])
        sums = sums + torch.stack(back[1:]).double()
    # two sums of n / 2 terms against one of n, each within `kn` of its terms' magnitudes
    size = torch.stack([(dy.float().abs() * ((x.float() - mean[:, None]) * rstd[:, None]).abs()).sum(0), dy.float().abs().sum(0)])
    kn = 2 * (64.0 + n / 256) * U
    assert bool(((torch.stack([dw, db]).double() - sums).abs() <= kn * size.double()).all())


def test_no_rows():
    x = torch.empty((0, 24), device=DEV)
    y, mean, rstd = bh.layer_norm(x)
    assert y.shape == (0, 24) and mean.numel() == rstd.numel() == 0
    dx, dw, db = bh.layer_norm_backward(x, x, vec(24, torch.float32, 1, 1.0, 0.1), mean, rstd)
    assert dx.shape == (0, 24) and bool((dw == 0).all()) and bool((db == 0).all())


def test_same_bits_again_on_another_stream_and_in_a_graph():
    n, d = 4001, 200
    x, dy = rows(n, d, torch.bfloat16, 1), rows(n, d, torch.bfloat16, 2)
    w, b = vec(d, torch.float32, 3, 1.0, 0.2), vec(d, torch.float32, 4, 0.0, 0.1)
    ws = torch.empty(bh.layer_norm_workspace_size(n, d), dtype=torch.uint8, device=DEV)

    def both():
        y, mean, rstd = bh.layer_norm(x, w, b)
        return (y, mean, rstd, *bh.layer_norm_backward(dy, x, w, mean, rstd, workspace=ws))

    want = [t.clone() for t in both()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        bh.layer_norm_backward(x, dy, w, want[1], want[2], workspace=ws)  # eager work on the same workspace
        torch.cuda.synchronize()


def test_refusals():
    x = rows(4, 8, torch.float32, 1)
    w, m = vec(8, torch.float32, 1, 1.0, 0.1), torch.zeros(4, device=DEV)
    for call in (lambda: bh.layer_norm(x.double()), lambda: bh.layer_norm(x.t()), lambda: bh.layer_norm(x, w[:7]),
                 lambda: bh.layer_norm(x, w, w.half()), lambda: bh.layer_norm(x, out=x[:, :7]),
                 lambda: bh.layer_norm(x, out=x.half()), lambda: bh.layer_norm_backward(x.half(), x, w, m, m),
                 lambda: bh.layer_norm_backward(x[:3], x, w, m, m), lambda: bh.layer_norm_backward(x, x, w, m[:3], m),
                 lambda: bh.layer_norm_backward(x, x, w, m.half(), m), lambda: bh.layer_norm_backward(x, x, w.cpu(), m, m)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(bh.BhtsneError) as e:
        bh.layer_norm(x, eps=-1.0)
    assert e.value.status == bh.BHTSNE_EINVAL
    with pytest.raises(bh.BhtsneError) as e:
        bh.layer_norm_backward(x, x, w, m, m, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == bh.BHTSNE_EWORKSPACE
    assert np.isfinite(float(bh.layer_norm(x)[0].sum()))
