"""Batches whose matrices lie between one another's rows, as a rows x batch x cols array holds them."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"


def between(batch, rows, cols, pad, values):
    """values (batch x rows x cols) as a view of rows x batch x (cols + pad), whose other elements are NaN."""
    buf = torch.full((rows, batch, cols + pad), float("nan"), dtype=values.dtype, device=DEV)
    view = buf.transpose(0, 1)[:, :, :cols]
    view.copy_(values)
    return buf, view


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("batch,rows,cols,pad", [(3, 20, 50, 0), (2, 300, 40, 3), (4, 96, 136, 0), (3, 130, 77, 1), (2, 1, 30, 2)])
def test_rows_between_rows(batch, rows, cols, pad, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    G, W, M = (torch.randn(batch, rows, cols, generator=g).to(t).to(DEV) for t in (dtype, dtype, torch.float32))
    want = bh.orthogonalise(G)
    _, Gv = between(batch, rows, cols, pad, G)
    buf, out = between(batch, rows, cols, pad, torch.zeros_like(G))
    assert bh.orthogonalise(Gv, out=out) is out and torch.equal(out, want)
    assert bool(torch.isnan(buf[:, :, cols:]).all())
    (wbuf, Wv), (mbuf, Mv) = between(batch, rows, cols, pad, W), between(batch, rows, cols, pad, M)
    bh.muon_step(W, G, M, 0.1)
    bh.muon_step(Wv, Gv, Mv, 0.1)
    assert torch.equal(Wv, W) and torch.equal(Mv, M)
    assert bool(torch.isnan(wbuf[:, :, cols:]).all()) and bool(torch.isnan(mbuf[:, :, cols:]).all())
