"""Tensors with a forward-mode tangent: the trained map's operators have no such derivative, and say so instead of losing it."""
import pytest
import torch
from torch.autograd import forward_ad as fw

import paper_2212_11506_amd as bh
from paper_2212_11506_amd import _binding as b


def test_arguments_with_a_tangent_are_refused():
    """On the host, where a tensor's device is -1."""
    x, v = torch.zeros(4, 8), torch.zeros(4)
    looks = [lambda t: b._rows(t, "x", t.shape, t.dtype, -1), lambda t: b._matrices(t, "x", t.shape, t.dtype, -1)]
    with fw.dual_level():
        for look in looks:
            look(x)
            with pytest.raises(ValueError, match="x has a tangent"):
                look(fw.make_dual(x, torch.ones(4, 8)))
        b._vector(v, "v", 4, -1)
        with pytest.raises(ValueError, match="v has a tangent"):
            b._vector(fw.make_dual(v, torch.ones(4)), "v", 4, -1)
        primal = fw.unpack_dual(fw.make_dual(x, torch.ones(4, 8))).primal
        looks[0](primal)


@pytest.mark.gpu
def test_calls_with_a_tangent_are_refused():
    n, d, f, v, k = 6, 8, 16, 20, 3
    g = torch.Generator().manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    x, gate, up, dh, z, u, w, y = make(n, d), make(f, d), make(f, d), make(n, f), make(n, v), make(n, k), make(d), make(n)
    idx = torch.arange(n * k, dtype=torch.int32).view(n, k).cuda()
    q, s = bh.quantise_rows(gate)
    calls = [(bh.gated_layer, [x, gate, up]), (bh.gated_layer_backward, [dh, x, gate, up, dh, dh]), (bh.quantise_rows, [x]), (bh.linear_i8, [x, q, s]),
             (bh.distil_loss, [z, idx, u]), (bh.distil_loss_backward, [y, z, idx, u, y]), (bh.layer_norm, [x, w, w]),
             (bh.layer_norm_backward, [x, x, w, y, y]), (bh.orthogonalise, [gate])]
    for call, given in calls:
        call(*given)
        for at, t in enumerate(given):
            if not t.is_floating_point():
                continue
            with fw.dual_level():
                call(*given)  # none has one
                dual = [fw.make_dual(p, torch.ones_like(p)) if i == at else p for i, p in enumerate(given)]
                with pytest.raises(ValueError, match="tangent"):
                    call(*dual)
                with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                    call(*dual)
    # recorded for reverse mode too: torch's own refusal
    with fw.dual_level(), pytest.raises((ValueError, NotImplementedError)):
        bh.gated_layer(fw.make_dual(x.requires_grad_(), torch.ones_like(x)), gate, up)
