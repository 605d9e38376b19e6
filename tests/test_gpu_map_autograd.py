"""The trained map's operators inside torch's graph: layer norm's gradient reaches what lies before it, what has none
refuses.

Tolerances of gradients: sums of n rows or d features in fp32, (64 + n / 256) 2^-24 of their terms as in the layer norm's
own tests; 1e-5 of the norm covers both at these sizes."""
import pytest
import torch
import torch.nn.functional as F

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gauss(*shape, seed=0, dtype=torch.float32, spread=1.0, mean=0.0):
    return (mean + spread * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


def rel(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


LOSSES = [("weighted", lambda y, r: (y * r).sum()), ("sum of squares", lambda y, r: y.square().sum()),
          ("one value for all", lambda y, r: (y + y.detach() * 0).sum() + (y * r).sum()),
          ("every other feature", lambda y, r: (y[:, ::2] * r[:, ::2]).sum()), ("rows' means", lambda y, r: (y.mean(1) * r[:, 0]).sum())]


@pytest.mark.parametrize("name,loss", LOSSES)
@pytest.mark.parametrize("with_weight", [True, False])
@pytest.mark.parametrize("with_bias", [True, False])
def test_gradients_reach_the_inputs(name, loss, with_weight, with_bias):
    n, d, k = 300, 70, 40
    x0, A, r = gauss(n, k, seed=1), gauss(k, d, seed=2, spread=0.2), gauss(n, d, seed=3)
    w, b = gauss(d, seed=4, spread=0.2, mean=1.0), gauss(d, seed=5)
    leaves = [A] + [w] * with_weight + [b] * with_bias
    for t in leaves:
        t.requires_grad_()
    y, mean, rstd = bh.layer_norm(x0 @ A, w if with_weight else None, b if with_bias else None)
    assert y.requires_grad and not mean.requires_grad and not rstd.requires_grad
    loss(y, r).backward()
    exact = [t.detach().double().cpu().requires_grad_() for t in leaves]
    rest = exact[1:]
    z = F.layer_norm(x0.double().cpu() @ exact[0], (d,), rest.pop(0) if with_weight else None, rest.pop(0) if with_bias else None, 1e-5)
    r64 = r.double().cpu()
    sizes = [g.norm() for g in torch.autograd.grad((z * r64).sum(), exact, retain_graph=True)]
    loss(z, r64).backward()
    for got, want, size in zip(leaves, exact, sizes):
        assert got.grad is not None and got.grad.dtype == got.dtype
        # a loss that the norm makes constant (rows' means without a weight) has a gradient of zero: against the weighted one's
        assert float((got.grad.double().cpu() - want.grad).norm()) <= 1e-5 * float(max(want.grad.norm(), size))


def test_a_bias_alone_keeps_its_type():
    x, b = gauss(500, 64, dtype=torch.bfloat16), gauss(64, seed=1).requires_grad_()
    y = bh.layer_norm(x, None, b)[0]
    r = gauss(500, 64, seed=2, dtype=torch.bfloat16)
    y.backward(r)
    assert b.grad.dtype == torch.float32 and rel(b.grad, r.double().cpu().sum(0)) <= 1e-6


def test_without_a_graph_there_is_none():
    x, w = gauss(8, 16), gauss(16, seed=1).requires_grad_()
    with torch.no_grad():
        y = bh.layer_norm(x, w)[0]
    assert not y.requires_grad
    assert not bh.layer_norm(x)[0].requires_grad
    with torch.inference_mode():
        z = bh.layer_norm(x, w)[0]
        bh.layer_norm(z, w, out=z)
    ones = torch.ones(8, 16, device=DEV)
    dx = bh.layer_norm_backward(ones, x, w, *bh.layer_norm(x, w)[1:])[0]
    assert not dx.requires_grad


def test_refusals_of_what_has_no_gradient():
    x, w = gauss(8, 16).requires_grad_(), gauss(16, seed=1)
    for call in (lambda: bh.layer_norm(x, w, out=torch.empty(8, 16, device=DEV)), lambda: bh.orthogonalise(x),
                 lambda: bh.orthogonalise(x, out=torch.empty(8, 16, device=DEV))):
        with pytest.raises(ValueError, match="gradient"):
            call()
    with torch.no_grad():
        assert bh.orthogonalise(x).shape == (8, 16)
    y = bh.layer_norm(x, w)[0]
    g, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):  # its gradient has none of its own
        g.sum().backward()


def test_a_step_of_weights_that_require_gradients():
    w, m = gauss(20, 30).requires_grad_(), torch.zeros(20, 30, device=DEV)
    (w * gauss(20, 30, seed=1)).sum().backward()
    before = w.detach().clone()
    bh.muon_step(w, w.grad, m, 0.1)
    assert w.is_leaf and w.requires_grad and not torch.equal(w.detach(), before)


def overwrites():
    x, w = gauss(8, 16, seed=7), gauss(16, seed=1)
    mean, rstd = bh.layer_norm(x, w)[1:]
    m = torch.zeros(8, 16, device=DEV)
    yield "out=", lambda t: bh.layer_norm(t, w, out=t)
    yield "dx=", lambda t: bh.layer_norm_backward(t, x, w, mean, rstd, dx=t)
    yield "orthogonalise", lambda t: bh.orthogonalise(t, out=t)
    yield "weights", lambda t: bh.muon_step(t, x, m.clone(), 0.1)
    yield "momentum", lambda t: bh.muon_step(x.clone(), x, t, 0.1)


def test_writing_in_place_is_known_to_the_graph():
    """A graph that has saved a tensor does not run backward on what has been written into it since."""
    for name, write in overwrites():
        t, v = gauss(8, 16, seed=3), gauss(8, 16, seed=4).requires_grad_()
        loss = (t * v).sum()  # saves t
        before = t._version
        with torch.no_grad():
            write(t)
        assert t._version > before, name
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        if name != "momentum":
            view = gauss(4, 8, 16, seed=5)
            with torch.no_grad():
                write(view[1])
            assert view._version > 0, name
