"""Every pair of types that rows and parameters can have, forward and backward, in rows of each kind of kernel."""
import pytest
import torch

import paper_2212_11506_amd as bh
from test_gpu_norm import check_backward, check_forward, rows, stats, vec

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("ptype", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d", [(1, 2), (37, 50), (37, 96), (700, 504), (5, 2000), (3, 9001), (2, 16_400), (2, 20_001)])
def test_types_of_rows_and_parameters(n, d, dtype, ptype):
    print(f"[norm] n={n} d={d} {dtype} {ptype}", flush=True)
    x, dy = rows(n, d, dtype, 1), rows(n, d, dtype, 2, 0, 0.1, 0.01)
    w, b = vec(d + 1, ptype, 3, 1.0, 0.2), vec(d + 1, ptype, 4, 0.0, 0.1)
    for i in (0, 1):  # aligned, and one element behind it
        for ww, bb in ((w[i:i + d], b[i:i + d]), (w[i:i + d], None), (None, b[i:i + d])):
            check_forward(x, ww, bb, bh.layer_norm(x, ww, bb, eps=1e-5))
        mean, rstd = stats(x)
        check_backward(dy, x, w[i:i + d], mean, rstd, bh.layer_norm_backward(dy, x, w[i:i + d], mean, rstd))
