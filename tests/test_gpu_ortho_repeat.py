"""The products' epilogues pass values between a wave's lanes through LDS; whatever the waves' timing, the same bits
come out, alone, in a batch and beside other work."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(65, 300), (130, 200), (500, 520), (1024, 1030), (1500, 700), (2048, 2100), (4000, 4160)])
def test_same_bits_again(shape, dtype):
    G = torch.randn(shape, generator=torch.Generator().manual_seed(shape[0])).to(dtype).to(DEV)
    # memory of its own before the first call: what that call frees is still in use on this stream
    side, other = torch.cuda.Stream(), torch.zeros(1 << 24, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    first = bh.orthogonalise(G)
    for k in range(3):
        with torch.cuda.stream(side):
            for _ in range(4):
                other.add_(1.0)
        assert torch.equal(bh.orthogonalise(G), first)
    torch.cuda.synchronize()
    if shape[0] <= 600:
        assert all(torch.equal(o, first) for o in bh.orthogonalise(G.expand(3, *shape))), "tiles may differ: values may not"
