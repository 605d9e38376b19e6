"""Which orders of a batch's matrices are taken where they are written: host-side, nothing is launched (a workspace that is
too small is refused last, so it shows that everything else was taken)."""
import ctypes as C

import pytest

import paper_2212_11506_amd as bh
from paper_2212_11506_amd._binding import _Matrices

FAKE = 1 << 20


def status(stride, batch_stride, batch=3, rows=70, cols=64, momentum=False):
    ok, x = _Matrices(FAKE, cols, rows * cols), _Matrices(FAKE, stride, batch_stride)
    lib = bh.load_library()
    if momentum:
        return lib.bhtsne_muon_step(C.byref(ok), C.byref(ok), C.byref(x), batch, rows, cols, 0, 0.1, 0.9, 1, 0.0, 1.0, None, 5,
                                    1e-7, FAKE, 8, None)
    return lib.bhtsne_orthogonalise(C.byref(ok), batch, rows, cols, 0, None, 5, 1e-7, C.byref(x), FAKE, 8, None)


@pytest.mark.parametrize("momentum", [False, True])
@pytest.mark.parametrize("stride,batch_stride,taken", [
    (64, 70 * 64, True), (64, 70 * 64 - 1, False), (80, 69 * 80 + 64, True), (80, 69 * 80 + 63, False),  # one behind the other
    (192, 64, True), (191, 64, False), (200, 68, True), (199, 68, False), (400, 68, True),               # rows between rows
    (192, 63, False), (64, 0, False), (192, 1 << 47, True), ((1 << 31) - 1, 1 << 29, True), ((1 << 31) - 1, 1 << 30, False)])
def test_orders(stride, batch_stride, taken, momentum):
    assert status(stride, batch_stride, momentum=momentum) == (bh.BHTSNE_EWORKSPACE if taken else bh.BHTSNE_EINVAL)


def test_sizes_are_refused_before_they_are_multiplied():
    for momentum in (False, True):
        assert status((1 << 31) - 1, 5, batch=2, rows=1 << 33, momentum=momentum) == bh.BHTSNE_EINVAL
        assert status((1 << 31) - 1, 5, batch=1 << 62, momentum=momentum) == bh.BHTSNE_EINVAL
