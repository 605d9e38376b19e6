"""Host-side checks of the trained map's operators that need no GPU: workspace sizes, and refusals before the
device is touched."""
import ctypes as C

import pytest
import torch

import paper_2212_11506_amd as bh
from paper_2212_11506_amd._binding import _Matrices

FAKE = 1 << 20  # a non-null, 256-aligned address that is never dereferenced on rejection
BIG = 1 << 50
INF, NAN = float("inf"), float("nan")


def _norm(**kw):
    a = dict(x=FAKE, xs=8, w=FAKE, b=FAKE, n=4, d=8, eps=1e-5, t=0, p=0, y=FAKE, ys=8, m=FAKE, r=FAKE) | kw
    return bh.load_library().bhtsne_layer_norm(a["x"], a["xs"], a["w"], a["b"], a["n"], a["d"], a["eps"], a["t"], a["p"],
                                               a["y"], a["ys"], a["m"], a["r"], None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(y=None), dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=(1 << 24) + 1),
                                 dict(xs=7), dict(xs=-8), dict(xs=1 << 31), dict(ys=0), dict(ys=7), dict(eps=-1e-9),
                                 dict(eps=NAN), dict(eps=INF), dict(t=3), dict(t=-1), dict(p=3), dict(x=FAKE + 2),
                                 dict(y=FAKE + 1), dict(w=FAKE + 2), dict(b=FAKE + 1), dict(m=FAKE + 2), dict(r=FAKE + 2)])
def test_layer_norm_refuses(bad):
    assert _norm(**bad) == bh.BHTSNE_EINVAL


def _back(**kw):
    a = dict(dy=FAKE, dys=8, x=FAKE, xs=8, w=FAKE, m=FAKE, r=FAKE, n=4, d=8, t=0, p=0, dx=FAKE, dxs=8, dw=FAKE, db=FAKE,
             ws=FAKE, wsb=BIG) | kw
    return bh.load_library().bhtsne_layer_norm_backward(a["dy"], a["dys"], a["x"], a["xs"], a["w"], a["m"], a["r"], a["n"],
                                                        a["d"], a["t"], a["p"], a["dx"], a["dxs"], a["dw"], a["db"],
                                                        a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(m=None), dict(r=None), dict(n=-1), dict(d=0), dict(dys=7),
                                 dict(xs=5), dict(dxs=0), dict(dx=None, dw=None, db=None), dict(t=9), dict(p=-1),
                                 dict(dx=FAKE + 2), dict(dw=FAKE + 1), dict(db=FAKE + 2), dict(dy=FAKE + 1)])
def test_layer_norm_backward_refuses(bad):
    assert _back(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(ws=None), dict(ws=FAKE + 128), dict(wsb=16)])
def test_layer_norm_backward_wants_its_workspace(bad):
    assert _back(**bad) == bh.BHTSNE_EWORKSPACE


def test_layer_norm_workspace_size():
    size = bh.layer_norm_workspace_size
    assert size(-1, 8) == size(4, 0) == size(1 << 31, 8) == size(4, (1 << 24) + 1) == 0
    assert size(0, 8) > 0 and size(1, 8) % 256 == 0
    assert size(10_000_000, 512) == size(1_300_000, 512) <= 16 << 20  # bounded by the chip, not by the rows


def _mat(data=FAKE, stride=64, batch_stride=64 * 64):
    return _Matrices(data, stride, batch_stride)


def _orth(**kw):
    a = dict(G=_mat(), O=_mat(), batch=1, rows=64, cols=64, t=0, coef=None, steps=5, eps=1e-7, ws=FAKE, wsb=BIG) | kw
    ref = lambda m: C.byref(m) if m is not None else None  # noqa: E731
    coef = (C.c_double * len(a["coef"]))(*a["coef"]) if a["coef"] else None
    return bh.load_library().bhtsne_orthogonalise(ref(a["G"]), a["batch"], a["rows"], a["cols"], a["t"], coef, a["steps"],
                                                  a["eps"], ref(a["O"]), a["ws"], a["wsb"], None)


BAD_MATRICES = [dict(rows=0), dict(cols=0), dict(batch=-1), dict(batch=65536), dict(rows=65537), dict(cols=65537), dict(t=3),
                dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=NAN)]


@pytest.mark.parametrize("bad", BAD_MATRICES + [
    dict(G=None), dict(O=None), dict(G=_mat(data=None)), dict(O=_mat(data=None)), dict(G=_mat(stride=63)), dict(O=_mat(stride=0)),
    dict(G=_mat(data=FAKE + 2)), dict(batch=2, O=_mat(batch_stride=64 * 64 - 1)), dict(batch=2, O=_mat(batch_stride=0)),
    dict(batch=2, G=_mat(batch_stride=-1)), dict(coef=[NAN, 0.0, 0.0], steps=1), dict(coef=[1.0, INF, 0.0], steps=1),
    dict(coef=[100.0, 0.0, 0.0], steps=1), dict(coef=[2.0, 0.0, 0.0] * 7, steps=7)])
def test_orthogonalise_refuses(bad):
    assert _orth(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(ws=None), dict(ws=FAKE + 64), dict(wsb=1024)])
def test_orthogonalise_wants_its_workspace(bad):
    assert _orth(**bad) == bh.BHTSNE_EWORKSPACE


def _muon(**kw):
    a = dict(W=_mat(), G=_mat(), M=_mat(), batch=1, rows=64, cols=64, t=0, lr=0.02, mu=0.95, wd=0.0, scale=1.0, steps=5,
             eps=1e-7, ws=FAKE, wsb=BIG) | kw
    ref = lambda m: C.byref(m) if m is not None else None  # noqa: E731
    return bh.load_library().bhtsne_muon_step(ref(a["W"]), ref(a["G"]), ref(a["M"]), a["batch"], a["rows"], a["cols"], a["t"],
                                              a["lr"], a["mu"], 1, a["wd"], a["scale"], None, a["steps"], a["eps"], a["ws"],
                                              a["wsb"], None)


@pytest.mark.parametrize("bad", BAD_MATRICES + [
    dict(W=None), dict(G=None), dict(M=None), dict(M=_mat(data=None)), dict(M=_mat(stride=10)), dict(M=_mat(data=FAKE + 2)),
    dict(batch=2, W=_mat(batch_stride=1)), dict(batch=2, M=_mat(batch_stride=1)), dict(lr=0.0), dict(lr=NAN), dict(lr=INF),
    dict(mu=1.0), dict(mu=-0.1), dict(mu=NAN), dict(wd=-0.1), dict(wd=INF), dict(scale=NAN)])
def test_muon_step_refuses(bad):
    assert _muon(**bad) == bh.BHTSNE_EINVAL


def test_muon_step_wants_its_workspace():
    assert _muon(ws=None) == _muon(wsb=8) == bh.BHTSNE_EWORKSPACE


def test_orthogonalise_workspace_size():
    size = bh.orthogonalise_workspace_size
    assert size(1, 0, 5) == size(1, 5, 0) == size(-1, 5, 5) == size(1, 65537, 1) == size(65536, 1, 1) == 0
    assert size(0, 5, 5) > 0 and size(1, 5, 7) % 256 == 0
    assert size(3, 100, 200) == 3 * size(1, 100, 200) == 3 * size(1, 200, 100)


def test_python_refuses_before_the_library_is_called():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        bh.layer_norm(x)  # not on the GPU
    with pytest.raises(ValueError):
        bh.layer_norm(torch.zeros(4, 8, 2))
    with pytest.raises(ValueError):
        bh.orthogonalise(x)
    with pytest.raises(ValueError):
        bh.orthogonalise(torch.zeros(8))
    with pytest.raises(ValueError):
        bh.muon_step(x, x, x, 0.1)
