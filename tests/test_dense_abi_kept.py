"""Host-side checks of the list loss' calls with what the backward pass keeps: no GPU."""
import pytest

import paper_2212_11506_amd as bh
from tests.test_dense_abi import A_, B_, BIG, FAKE, LISTS, W_, X_, call

D_, E_ = FAKE + 4096 * 5, FAKE + 4096 * 6


def distil(**bad):
    return call("bhtsne_distil_loss_kept", "z zs n v i is_ u us k T t ut l e kept ws wsb",
                dict(z=FAKE, zs=50_000, n=2, v=50_000, i=X_, is_=5, u=A_, us=5, k=5, T=1.0, t=0, ut=0, l=B_, e=W_, kept=D_, ws=E_, wsb=BIG), bad)


@pytest.mark.parametrize("bad", LISTS + [dict(l=None, e=None, kept=None), dict(l=B_ + 1), dict(e=W_ + 2), dict(kept=D_ + 2)])
def test_distil_loss_kept_refuses(bad):
    assert distil(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(ws=None), dict(ws=E_ + 128), dict(wsb=64)])
def test_distil_loss_kept_wants_its_workspace_for_long_rows(bad):
    assert distil(**bad) == bh.BHTSNE_EWORKSPACE


def distil_back(**bad):
    return call("bhtsne_distil_loss_backward_kept", "dl z zs n v i is_ u us k e kept T t ut dz dzs",
                dict(dl=B_, z=FAKE, zs=50_000, n=2, v=50_000, i=X_, is_=5, u=A_, us=5, k=5, e=W_, kept=D_, T=1.0, t=0, ut=0, dz=E_, dzs=50_000), bad)


@pytest.mark.parametrize("bad", LISTS + [dict(dl=None), dict(e=None), dict(dl=B_ + 2), dict(e=W_ + 1), dict(kept=D_ + 2), dict(dz=None), dict(dzs=49_999),
                                         dict(dz=E_ + 2)])
def test_distil_loss_backward_kept_refuses(bad):
    assert distil_back(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(l=W_), dict(l=D_), dict(e=D_), dict(l=FAKE), dict(e=FAKE), dict(kept=FAKE), dict(l=X_), dict(e=X_), dict(l=A_),
                                 dict(kept=A_), dict(l=E_), dict(kept=E_)])
def test_distil_loss_refuses_outputs_at_one_address(bad):
    assert distil(**bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("bad", [dict(dz=B_), dict(dz=W_), dict(dz=D_), dict(dz=X_), dict(dz=A_), dict(dz=FAKE, dzs=50_001), dict(dz=FAKE, zs=50_001),
                                 dict(dz=FAKE, zs=0)])
def test_distil_loss_backward_refuses_outputs_over_inputs(bad):
    """Blocks would write rows that others have still to read."""
    assert distil_back(**bad) == bh.BHTSNE_EINVAL


def test_the_calls_without_kept_refuse_them_too():
    args = dict(z=FAKE, zs=50_000, n=2, v=50_000, i=X_, is_=5, u=A_, us=5, k=5, T=1.0, t=0, ut=0, l=B_, e=W_, ws=E_, wsb=BIG)
    for bad in (dict(l=W_), dict(e=FAKE), dict(e=A_)):
        assert call("bhtsne_distil_loss", "z zs n v i is_ u us k T t ut l e ws wsb", args, bad) == bh.BHTSNE_EINVAL
    args = dict(dl=B_, z=FAKE, zs=50_000, n=2, v=50_000, i=X_, is_=5, u=A_, us=5, k=5, e=W_, T=1.0, t=0, ut=0, dz=E_, dzs=50_000)
    for bad in (dict(dz=FAKE, zs=0), dict(dz=W_), dict(dz=B_)):
        assert call("bhtsne_distil_loss_backward", "dl z zs n v i is_ u us k e T t ut dz dzs", args, bad) == bh.BHTSNE_EINVAL


@pytest.mark.parametrize("good", [dict(dz=FAKE, n=0, zs=0), dict(dz=B_, n=0), dict(dl=None, e=None, n=0)])
def test_no_rows_overlap_nothing(good):
    assert distil_back(**good) != bh.BHTSNE_EINVAL
