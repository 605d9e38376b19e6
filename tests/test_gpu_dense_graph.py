"""What the nodes of torch's graph hold and fill in a backward pass."""
import pytest
import torch

import paper_2212_11506_amd as bh
from paper_2212_11506_amd import _binding as b
from tests.test_gpu_distil import case
from tests.test_gpu_gated import mat

pytestmark = pytest.mark.gpu
DEV = "cuda"


def nodes(dtype=torch.float32):
    """Each node's class, its leaves and a call that gives its differentiable output."""
    x, gate, up = (mat(*s, dtype, k).requires_grad_() for k, s in enumerate([(50, 24), (30, 24), (30, 24)]))
    z, idx, u = case(50, 200, 7, dtype, 3)
    z = z.clone().requires_grad_()
    w, shift = torch.ones(24, dtype=dtype, device=DEV).requires_grad_(), torch.zeros(24, dtype=dtype, device=DEV).requires_grad_()
    return [(b._GatedLayer, (x, gate, up), lambda: bh.gated_layer(x, gate, up, keep=True)[0]),
            (b._DistilLoss, (z,), lambda: bh.distil_loss(z, idx, u)[0]),
            (b._LayerNorm, (x, w, shift), lambda: bh.layer_norm(x, w, shift)[0])]


@pytest.mark.parametrize("which", range(3))
def test_no_gradients_of_what_has_none(which, monkeypatch):
    node, leaves, call = nodes()[which]
    seen, backward = [], node.backward
    monkeypatch.setattr(node, "backward", staticmethod(lambda ctx, *grads: (seen.append(grads), backward(ctx, *grads))[1]))
    call().sum().backward()
    (grads,) = seen
    assert isinstance(grads[0], torch.Tensor) and all(g is None for g in grads[1:])
    assert all(t.grad is not None for t in leaves)


class Stop(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y):
        return y.clone()

    @staticmethod
    def backward(ctx, _):
        return None


@pytest.mark.parametrize("which", range(3))
def test_no_gradient_comes_back(which):
    _, leaves, call = nodes()[which]
    Stop.apply(call()).sum().backward()
    assert all(t.grad is None or not t.grad.any() for t in leaves)


def test_memory_of_a_backward_pass():
    """The operands in the workspace, the sum's gradient laid out (one value for all: n f values) and the results; a's and b's
    gradients of zeros would be 2 n f values more."""
    n, d, f, t = 20_000, 16, 2048, torch.bfloat16
    x, gate, up = (mat(*s, t, k).requires_grad_() for k, s in enumerate([(n, d), (f, d), (f, d)]))
    total = bh.gated_layer(x, gate, up).sum()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    total.backward()
    more = torch.cuda.max_memory_allocated() - before
    # rounded up to the allocator's blocks: half an array is room for them and for the gradients
    assert more <= bh.gated_layer_workspace_size(n, d, f, t) + n * f * 2 + n * f * 2 // 2


def test_outputs_that_torch_records_are_refused():
    """What is written over a recorded tensor is not in its graph, whose gradients would be those of the values before."""
    x, gate, up = (mat(*s, torch.float32, k) for k, s in enumerate([(5, 24), (30, 24), (30, 24)]))
    w, ws = bh.quantise_rows(gate)
    calls = [lambda out: bh.gated_layer(x, gate, up, out=out), lambda out: bh.gated_layer(x, gate, up, "gelu", keep=True, out=out)[0],
             lambda out: bh.linear_i8(x, w, ws, out=out)]
    leaf = torch.zeros(5, 30, device=DEV).requires_grad_()
    for call in calls:
        for out in (leaf, leaf * 2):
            before = out.detach().clone()
            with pytest.raises(ValueError, match="gradient"):
                call(out)
            assert torch.equal(out.detach(), before)
            with torch.no_grad():
                assert call(out) is out
                leaf.zero_()
