"""Host-side checks of the trained map's dense operators that need no GPU: workspace sizes, and refusals before the device
is touched."""
import pytest
import torch

import paper_2212_11506_amd as bh
from paper_2212_11506_amd import _binding as b
from tests.test_map_binding import Elsewhere

FAKE = 1 << 20  # non-null, 256-aligned addresses that are never dereferenced on rejection
X_, A_, B_, W_ = (FAKE + 4096 * k for k in range(1, 5))
BIG = 1 << 50
INF, NAN = float("inf"), float("nan")


def call(name, order, given, bad):
    assert set(bad) <= set(given)
    a = given | bad
    return getattr(bh.load_library(), name)(*[a[k] for k in order.split()], None)


def gated(**bad):
    return call("bhtsne_gated_layer", "x xs g gs u us n d f act t h hs a as_ b bs",
                dict(x=FAKE, xs=8, g=FAKE, gs=8, u=FAKE, us=8, n=4, d=8, f=16, act=0, t=0, h=X_, hs=16, a=A_, as_=16, b=B_, bs=16), bad)


LAYER = [dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=65537), dict(f=0), dict(f=65537), dict(act=2), dict(act=-1), dict(t=3), dict(t=-1), dict(x=None),
         dict(xs=7), dict(xs=-8), dict(xs=1 << 31), dict(g=None), dict(gs=0), dict(gs=7), dict(u=None), dict(us=7), dict(us=1 << 31),
         dict(x=FAKE + 2), dict(g=FAKE + 1), dict(u=FAKE + 2), dict(as_=15), dict(bs=0), dict(a=FAKE + 1), dict(b=FAKE + 2)]


@pytest.mark.parametrize("bad", LAYER + [dict(h=None), dict(hs=15), dict(hs=0), dict(h=FAKE + 2), dict(h=FAKE), dict(a=FAKE), dict(h=A_), dict(a=B_)])
def test_gated_layer_refuses(bad):
    assert gated(**bad) == bh.BHTSNE_EINVAL


def gated_back(**bad):
    return call("bhtsne_gated_layer_backward", "dh dhs x xs g gs u us a as_ b bs n d f act t dx dxs dg dgs du dus ws wsb",
                dict(dh=FAKE, dhs=16, x=FAKE, xs=8, g=FAKE, gs=8, u=FAKE, us=8, a=FAKE, as_=16, b=FAKE, bs=16, n=4, d=8, f=16, act=0, t=0, dx=X_, dxs=8,
                     dg=A_, dgs=8, du=B_, dus=8, ws=FAKE, wsb=BIG), bad)


@pytest.mark.parametrize("bad", [c for c in LAYER if c != dict(bs=0)] + [
    dict(dh=None), dict(a=None), dict(b=None), dict(dhs=15), dict(bs=15), dict(dxs=7), dict(dxs=0), dict(dgs=7), dict(dus=0),
    dict(dx=FAKE + 1), dict(dg=FAKE + 2), dict(du=FAKE + 3), dict(dx=None, dg=None, du=None), dict(dx=FAKE), dict(dg=FAKE),
    dict(dx=A_), dict(dg=B_)])
def test_gated_layer_backward_refuses(bad):
    assert gated_back(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(ws=None), dict(ws=FAKE + 128), dict(wsb=64)])
def test_gated_layer_backward_wants_its_workspace(bad):
    assert gated_back(**bad) == bh.BHTSNE_EWORKSPACE


def test_gated_layer_workspace_size():
    size = bh.gated_layer_workspace_size
    assert size(-1, 8, 8) == size(4, 0, 8) == size(4, 8, 0) == size(1 << 31, 8, 8) == size(4, 65537, 8) == size(4, 8, 65537) == 0
    assert size(0, 8, 8) > 0 and size(5, 7, 9) % 256 == 0
    assert size(1000, 500, 600, torch.float32) > size(1000, 500, 600, torch.float16) == size(1000, 500, 600, torch.bfloat16)
    # few outputs: operands of 32 bits for every type
    assert size(1000, 50, 60, torch.float16) == size(1000, 50, 60, torch.bfloat16) >= (2 * 1000 * 60 + 2 * 60 * 50) * 4


def quantise(**bad):
    return call("bhtsne_quantise_rows", "x xs n d t q qs s", dict(x=FAKE, xs=8, n=4, d=8, t=0, q=X_, qs=8, s=A_), bad)


@pytest.mark.parametrize("bad", [dict(x=None), dict(xs=7), dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=131072), dict(t=3), dict(q=None), dict(qs=7),
                                 dict(s=None), dict(s=FAKE + 2), dict(x=FAKE + 2), dict(q=FAKE), dict(s=X_)])
def test_quantise_rows_refuses(bad):
    assert quantise(**bad) == bh.BHTSNE_EINVAL


def linear(**bad):
    return call("bhtsne_linear_i8", "x xs xt xsc w ws_ wsc bias n d f t bt out os ws wsb",
                dict(x=FAKE, xs=8, xt=0, xsc=None, w=FAKE, ws_=8, wsc=FAKE, bias=FAKE, n=100, d=8, f=16, t=0, bt=0, out=X_, os=16, ws=FAKE, wsb=BIG), bad)


@pytest.mark.parametrize("bad", [dict(x=None), dict(xs=7), dict(xt=4), dict(xt=-1), dict(xsc=FAKE), dict(xt=3), dict(xt=3, xsc=FAKE + 1), dict(w=None),
                                 dict(ws_=0), dict(ws_=7), dict(wsc=None), dict(wsc=FAKE + 2), dict(bias=FAKE + 1), dict(n=-1), dict(d=0),
                                 dict(d=131072), dict(f=0), dict(f=1 << 31), dict(t=3), dict(bt=1), dict(t=1, bt=2), dict(out=None), dict(os=15),
                                 dict(out=FAKE + 1), dict(x=FAKE + 2), dict(out=FAKE)])
def test_linear_i8_refuses(bad):
    assert linear(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(ws=None), dict(ws=FAKE + 128), dict(wsb=64)])
def test_linear_i8_wants_its_workspace(bad):
    assert linear(**bad) == bh.BHTSNE_EWORKSPACE


def test_linear_i8_refuses_features_beyond_a_launch():
    for n in (1, 100):
        assert linear(n=n, f=(1 << 26) + 1, os=1 << 30) == bh.BHTSNE_EINVAL


def test_linear_i8_workspace_size():
    size = bh.linear_i8_workspace_size
    assert size(-1, 8) == size(4, 0) == size(4, 131072) == 0 and size(0, 8) > 0
    assert size(100, 20) >= 100 * 32 + 400 and size(100, 20) % 256 == 0
    assert size(1, 8192) == size(16, 512) == size(4, 1) == 256 < size(1, 8193) and size(17, 8) > 256 and size(16, 513) > 256


def distil(**bad):
    return call("bhtsne_distil_loss", "z zs n v i is_ u us k T t ut l e ws wsb",
                dict(z=FAKE, zs=50_000, n=2, v=50_000, i=FAKE, is_=5, u=FAKE, us=5, k=5, T=1.0, t=0, ut=0, l=FAKE, e=FAKE, ws=FAKE, wsb=BIG), bad)


LISTS = [dict(z=None), dict(zs=49_999), dict(zs=1 << 31), dict(n=-1), dict(n=1 << 31), dict(v=0), dict(v=1 << 31), dict(i=None), dict(is_=4), dict(u=None),
         dict(us=4), dict(k=-1), dict(k=2049, is_=4000, us=4000), dict(T=0.0), dict(T=-1.0), dict(T=NAN), dict(T=INF), dict(T=1e-7), dict(T=1e7),
         dict(t=3), dict(ut=3), dict(ut=1), dict(t=1, ut=2), dict(z=FAKE + 2), dict(i=FAKE + 2), dict(u=FAKE + 1)]


@pytest.mark.parametrize("bad", LISTS + [dict(l=None, e=None), dict(l=FAKE + 1), dict(e=FAKE + 2)])
def test_distil_loss_refuses(bad):
    assert distil(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(ws=None), dict(ws=FAKE + 128), dict(wsb=64)])
def test_distil_loss_wants_its_workspace_for_long_rows(bad):
    assert distil(**bad) == bh.BHTSNE_EWORKSPACE


def distil_back(**bad):
    return call("bhtsne_distil_loss_backward", "dl z zs n v i is_ u us k e T t ut dz dzs",
                dict(dl=FAKE, z=FAKE, zs=50_000, n=2, v=50_000, i=FAKE, is_=5, u=FAKE, us=5, k=5, e=FAKE, T=1.0, t=0, ut=0, dz=FAKE, dzs=50_000), bad)


@pytest.mark.parametrize("bad", LISTS + [dict(dl=None), dict(e=None), dict(dl=FAKE + 2), dict(e=FAKE + 1), dict(dz=None), dict(dzs=49_999), dict(dz=FAKE + 2)])
def test_distil_loss_backward_refuses(bad):
    assert distil_back(**bad) == bh.BHTSNE_EINVAL


def test_distil_loss_workspace_size():
    size = bh.distil_loss_workspace_size
    assert size(-1, 8) == size(4, 0) == size(1 << 31, 8) == 0
    assert size(100_000, 8) == size(1_000_000, 1000) == 256 < size(1, 1_300_000)
    assert size(1, (1 << 31) - 1) <= 1 << 20  # bounded by the chip


X, W, V, N = (4, 8), (16, 8), (16,), (4,)


def calls(at):
    h, lists, f32, i8, i32 = (4, 16), (4, 3), torch.float32, torch.int8, torch.int32
    return [lambda: b.gated_layer(at(0, X), at(1, W), at(2, W), out=at(3, h)),
            lambda: b.gated_layer_backward(at(0, h), at(1, X), at(2, W), at(3, W), at(4, h), at(5, h)),
            lambda: b.quantise_rows(at(0, X)),
            lambda: b.linear_i8(at(0, X), at(1, W, i8), at(2, V), bias=at(3, V), out=at(4, h)),
            lambda: b.linear_i8(at(0, X, i8), at(1, W, i8), at(2, V), at(3, N)),
            lambda: b.distil_loss(at(0, X), at(1, lists, i32), at(2, lists)),
            lambda: b.distil_loss_backward(at(0, N), at(1, X), at(2, lists, i32), at(3, lists), at(4, N), dlogits=at(5, X))]


COUNTS = [4, 6, 1, 5, 4, 3, 6]


@pytest.mark.parametrize("which", range(6))
def test_tensors_of_another_gpu_are_refused(which, monkeypatch):
    monkeypatch.setattr(b, "_current_gpu", lambda: 0)
    for name in ("gated_layer_workspace_size", "linear_i8_workspace_size", "distil_loss_workspace_size"):
        monkeypatch.setattr(b, name, lambda *a: 4096)

    class Library:
        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")

    monkeypatch.setattr(b, "load_library", Library)
    for run, count in zip(calls(lambda k, shape, dtype=torch.float32: Elsewhere(shape, 1 if k == which else 0, dtype)), COUNTS):
        if which < count:
            with pytest.raises(ValueError, match="GPU 1"):
                run()


def test_a_call_runs_on_the_current_gpu(monkeypatch):
    monkeypatch.setattr(b, "_current_gpu", lambda: 1)
    for run in calls(lambda k, shape, dtype=torch.float32: Elsewhere(shape, 0, dtype)):
        with pytest.raises(ValueError, match="current"):
            run()


def test_python_refuses_before_the_library_is_called():
    x, w = torch.zeros(4, 8), torch.zeros(16, 8)
    for run in (lambda: bh.gated_layer(x, w, w), lambda: bh.gated_layer(x, w, w, "relu"), lambda: bh.gated_layer(x, w[0], w), lambda: bh.quantise_rows(x),
                lambda: bh.quantise_rows(x[0]), lambda: bh.linear_i8(x, w.to(torch.int8), torch.zeros(16)), lambda: bh.linear_i8(x[0], w, w),
                lambda: bh.distil_loss(x, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)), lambda: bh.distil_loss(x[0], x, x),
                lambda: bh.distil_loss(x, x, x.double())):
        with pytest.raises(ValueError):
            run()
