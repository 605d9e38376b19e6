"""The dense operators as a program calls them: together, on another stream, captured and replayed, over arrays that 32-bit
offsets do not reach."""
import math

import pytest
import torch
import torch.nn.functional as F

import paper_2212_11506_amd as bh
from tests.test_gpu_distil import case as lists
from tests.test_gpu_distil import check_backward as check_lists_backward
from tests.test_gpu_distil import check_forward as check_lists
from tests.test_gpu_gated import check_forward, mat, operands
from tests.test_gpu_linear8 import check, ints, quantise64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def say(*a):
    print(*a, flush=True)


def every(x, gate, up, dh, w, ws, idx, u, workspaces=(None, None, None)):
    """Each operator once, on 16-bit points."""
    h, a, b = bh.gated_layer(x, gate, up, "gelu", keep=True)
    grads = bh.gated_layer_backward(dh, x, gate, up, a, b, "gelu", workspace=workspaces[0])
    q, s = bh.quantise_rows(h)
    out = bh.linear_i8(h, w, ws, workspace=workspaces[1])
    again = bh.linear_i8(q, w, ws, s)
    loss, lse = bh.distil_loss(out, idx, u, 2.0, workspace=workspaces[2])
    dz = bh.distil_loss_backward(torch.ones_like(loss), out, idx, u, lse, 2.0)
    return [h, a, b, *grads, q, s, out, again, loss, lse, dz]


def inputs(n, d, f, v, k, seed=0, dtype=torch.bfloat16):
    dh, x, gate, up, _, _ = operands(n, d, f, dtype)
    if seed:
        x, dh = x * (1 + seed) + seed / 8, dh * (2 + seed)
    w, ws = bh.quantise_rows(mat(v, f, dtype, 7, 0, f ** -0.5))
    idx, u = lists(n, v, k, dtype, 3 + seed)[1:]
    return x, gate, up, dh, w, ws, idx, u


@pytest.mark.parametrize("n,d,f,v,k", [(5, 64, 96, 40, 7), (300, 50, 200, 1000, 30), (3, 128, 256, 60_000, 20), (2500, 264, 2100, 300, 12)])
def test_on_another_stream(n, d, f, v, k):
    given = inputs(n, d, f, v, k)
    want = every(*given)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)  # what is not ordered behind this stream's work would read too early
        fresh = [t.clone() for t in given]
        got = every(*fresh)
    side.synchronize()
    for k_, (p, q) in enumerate(zip(got, want)):
        assert torch.equal(p, q), k_


@pytest.mark.parametrize("n,d,f,v,k", [(5, 64, 96, 40, 7), (300, 50, 200, 1000, 30), (3, 128, 256, 60_000, 20), (2500, 264, 2100, 300, 12)])
@pytest.mark.parametrize("own_workspaces", [False, True])
def test_captured_and_replayed(n, d, f, v, k, own_workspaces):
    """Every replay gives what the eager calls give on its inputs, with eager work and synchronisations between replays."""
    sets = [inputs(n, d, f, v, k, seed) for seed in range(3)]
    wants = [every(*s) for s in sets]
    spaces = (None, None, None)
    if own_workspaces:
        sizes = (bh.gated_layer_workspace_size(n, d, f, torch.bfloat16), bh.linear_i8_workspace_size(n, f), bh.distil_loss_workspace_size(n, v))
        spaces = tuple(torch.empty(s, dtype=torch.uint8, device=DEV) for s in sizes)
    given = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = every(*given, spaces)
    for turn in (1, 0, 2, 2, 1):
        for to, value in zip(given, sets[turn]):
            to.copy_(value)
        graph.replay()
        torch.cuda.synchronize()
        for k_, (p, q) in enumerate(zip(got, wants[turn])):
            assert torch.equal(p, q), (turn, k_)
        every(*sets[0])
        torch.randn(1000, device=DEV).sum().item()


def test_a_map_in_training():
    """Layer norms, gated layers and a head trained on neighbours' similarities: the gradients of all weights against the same
    map in 64 bits, then one step along them."""
    n, k = 600, 15
    x = torch.randn(n, 20, generator=torch.Generator().manual_seed(1)).to(DEV)
    dist = torch.cdist(x, x)
    dist.fill_diagonal_(float("inf"))
    near, idx = torch.topk(dist, k, largest=False)
    idx, near = idx.to(torch.int32).contiguous(), near.contiguous()
    sigma2 = bh.affinities(idx, near, 5.0, sigma2=True)[1]
    u = (-near.double().square() / (2.0 * sigma2[:, None])).float()
    gate, up, scale, shift, head = (t.clone().requires_grad_() for t in (
        mat(64, 20, torch.float32, 2, 0, 20 ** -0.5), mat(64, 20, torch.float32, 3, 0, 20 ** -0.5), torch.ones(64, device=DEV),
        torch.zeros(64, device=DEV), mat(n, 64, torch.float32, 4, 0, 0.1)))
    h = bh.layer_norm(bh.gated_layer(x, gate, up, "gelu"), scale, shift)[0]
    loss, _ = bh.distil_loss(h @ head.t(), idx, u)
    loss.mean().backward()
    leaves = [t.detach().double().cpu().requires_grad_() for t in (gate, up, scale, shift, head)]
    x64 = x.double().cpu()
    z = F.layer_norm(F.gelu(x64 @ leaves[0].t()) * (x64 @ leaves[1].t()), (64,), leaves[2], leaves[3], 1e-5) @ leaves[4].t()
    t = torch.softmax(u.double().cpu(), 1)
    want = (t * (t.log() - torch.log_softmax(z, 1).gather(1, idx.cpu().long()))).sum(1)
    # sums of 600 points and 64 features in fp32 through three layers
    assert float((loss.detach().double().cpu() - want.detach()).abs().max()) <= 1e-4 * float(want.detach().max())
    want.mean().backward()
    for got, exact in zip((gate, up, scale, shift, head), leaves):
        assert float((got.grad.double().cpu() - exact.grad).norm()) <= 1e-4 * float(exact.grad.norm())
    before = float(loss.detach().mean())
    with torch.no_grad():
        for w in (gate, up, head):
            bh.muon_step(w, w.grad, torch.zeros_like(w), 0.02)
        after = bh.distil_loss(bh.layer_norm(bh.gated_layer(x, gate, up, "gelu"), scale, shift)[0] @ head.t(), idx, u)[0]
        assert bool(after.isfinite().all()) and float(after.mean()) != before
        # the head in 8 bits: each logit off by half a step of its row and of its feature's weights, 64 times
        q, s = bh.quantise_rows(head)
        hidden = bh.layer_norm(bh.gated_layer(x, gate, up, "gelu"), scale, shift)[0]
        got = bh.linear_i8(hidden, q, s)
        exact = hidden.double() @ head.double().t().contiguous()
        step = hidden.abs().amax(1).double() / 127
        tol = 0.51 * (step[:, None] * head.double().abs().sum(1) + s.double() * hidden.double().abs().sum(1, keepdim=True) + 64 * step[:, None] * s.double())
        assert bool(((got.double() - exact).abs() <= tol).all())


def gaps(n, width, stride, dtype, seed):
    """n rows `stride` apart of an array that is not otherwise written."""
    buf = torch.empty(n * stride, dtype=dtype, device=DEV)
    out = buf.view(n, stride)[:, :width]
    out.copy_(mat(n, width, dtype, seed))
    return out


@pytest.mark.parametrize("n,d,f,stride", [(5, 200, 100, 1 << 30), (40, 50, 70, 1 << 27), (40, 203, 70, 1 << 27), (2600, 2056, 2050, 1 << 21)])
def test_offsets_beyond_32_bits(n, d, f, stride):
    t = torch.bfloat16
    say(f"[calls] rows {stride} apart, {n * stride / 2 ** 31:.1f} x 2^31 values")
    x, gate, up = gaps(n, d, stride, t, 1), mat(f, d, t, 2, 0, d ** -0.5), mat(f, d, t, 3, 0, d ** -0.5)
    h = gaps(n, f, stride, t, 4)
    bh.gated_layer(x, gate, up, out=h)
    check_forward(x, gate, up, "silu", h, None, None)
    near = x.contiguous()
    assert torch.equal(bh.gated_layer(near, gate, up), h)
    _, a, b = bh.gated_layer(near, gate, up, keep=True)
    dh = mat(n, f, t, 5, 0, 0.1)
    for p, q in zip(bh.gated_layer_backward(dh, x, gate, up, a, b), bh.gated_layer_backward(dh, near, gate, up, a, b)):
        assert torch.equal(p, q)
    w, ws = bh.quantise_rows(gate)
    bh.linear_i8(x, w, ws, out=h)
    check(*quantise64(near), w, ws, None, h)
    idx, u = lists(n, d, 9, t, 3)[1:]
    loss, lse = bh.distil_loss(x, idx, u)
    check_lists(x, idx, u, 1.0, (loss, lse))  # the order of a row's sum goes by its alignment
    assert torch.equal(torch.stack([loss, lse]), torch.stack(bh.distil_loss(x, idx, u)))
    dz = bh.distil_loss_backward(loss, near, idx, u, lse)
    bh.distil_loss_backward(loss, x, idx, u, lse, dlogits=x)
    assert torch.equal(x, dz)


def test_a_backward_pass_whose_operands_pass_32_bits():
    """da and db of more than 2^31 values."""
    n, d, f, t = 140_000, 64, 8192, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(1)
    make = lambda *s, by=1.0: (by * torch.randn(s, generator=g, device=DEV)).to(t)  # noqa: E731
    x, gate, up, dh, a, b = make(n, d), make(f, d, by=0.125), make(f, d, by=0.125), make(n, f, by=0.1), make(n, f), make(n, f)
    dx, dgate, dup = bh.gated_layer_backward(dh, x, gate, up, a, b)
    rows = torch.cat([torch.arange(50), torch.arange(n - 50, n)]).to(DEV)
    part = bh.gated_layer_backward(dh[rows], x[rows], gate, up, a[rows], b[rows])[0]
    # a point's sums, in other tiles: 2 f terms of operands alike, an output's rounding each
    assert bool(((dx[rows].double() - part.double()).abs() <= 2.0 ** -7 * part.double().abs() + 2 * f * 2.0 ** -24 * 0.2 * 8).all())
    want = torch.zeros(2, f, d, dtype=torch.float64, device=DEV)
    for i in range(0, n, 10_000):
        s = slice(i, i + 10_000)
        sg = torch.sigmoid(a[s].double())
        da, db = dh[s].double() * b[s].double() * sg * (1 + a[s].double() * (1 - sg)), dh[s].double() * a[s].double() * sg
        want[0] += da.T.contiguous() @ x[s].double()
        want[1] += db.T.contiguous() @ x[s].double()
    for got, exact in zip((dgate, dup), want):
        # operands rounded to 2^-8 at most, independently: their errors add up as the terms do; and the output's rounding
        assert float((got.double() - exact).norm() / exact.norm()) <= 2 * 2.0 ** -8


def test_lists_over_rows_that_pass_32_bits():
    n, v, k, t = 3, (1 << 30) + 7, 12, torch.float16
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.empty(n, v, dtype=t, device=DEV)
    for r in range(n):
        z[r] = torch.randn(v, generator=g, device=DEV, dtype=t)
    idx = torch.randint(v, (n, k), generator=g, device=DEV)
    idx[:, 0], idx[:, 1] = v - 1, v - 2
    idx = idx.to(torch.int32)
    u = -torch.rand(n, k, generator=g, device=DEV)
    loss, lse = bh.distil_loss(z, idx, u)
    for r in range(n):
        total = torch.zeros((), dtype=torch.float64, device=DEV)
        for i in range(0, v, 1 << 27):
            total += z[r, i:i + (1 << 27)].float().exp().sum(dtype=torch.float64)
        exact = float(total.log())
        # a lane's 2^30 / (683 x 256) terms in fp32, all of one sign
        assert abs(float(lse[r]) - exact) <= 6200 * 2.0 ** -24 + 2.0 ** -23 * exact
        shares = torch.softmax(u[r].double(), 0)
        want = float((shares * (shares.log() - z[r, idx[r].long()].double() + exact)).sum())
        assert abs(float(loss[r]) - want) <= 1e-3
    dz = bh.distil_loss_backward(torch.ones(n, device=DEV), z, idx, u, lse)
    for r in range(n):
        at = idx[r].long()
        shares = torch.softmax(u[r].double(), 0)
        assert float((dz[r, at].double() + shares).abs().max()) <= 1e-3 * 2
        for spot in (0, 12345, 1 << 29, v - 3):
            if not bool((at == spot).any()):
                assert abs(float(dz[r, spot]) - math.exp(float(z[r, spot]) - float(lse[r]))) <= 2.0 ** -24


def test_a_graph_of_lists_in_another_type():
    z, idx, u = lists(64, 3000, 20, torch.float16, 4)
    leaf = z.clone().requires_grad_()
    bh.distil_loss(leaf, idx, u, 0.5)[0].sum().backward()
    lse = bh.distil_loss(z, idx, u, 0.5)[1]
    check_lists_backward(torch.ones(64, device=DEV), z, idx, u, lse, 0.5, leaf.grad)


def test_ints_of_a_wider_array():
    w, ws = ints(33, 70, 2, 9), torch.ones(33, device=DEV)
    q = ints(50, 70, 3, 5)
    out = bh.linear_i8(q, w, ws, torch.ones(50, device=DEV))
    assert torch.equal(out.double(), q.double() @ w.double().T.contiguous())


def test_a_loss_changed_in_place():
    z, idx, u = lists(70, 400, 9, torch.float32, 8)
    scale = torch.rand(70, device=DEV) + 0.5
    leaf = z.clone().requires_grad_()
    loss, lse = bh.distil_loss(leaf, idx, u)
    kept = lse.clone()
    loss.mul_(scale)
    loss.sum().backward()
    assert torch.equal(lse, kept) and torch.equal(leaf.grad, bh.distil_loss_backward(scale, z, idx, u, kept))


@pytest.mark.parametrize("n", [3, 70, 900])
def test_a_captured_training_step(n):
    """Forward and backward of all nodes in one graph, replayed on other points, against the eager pass."""
    d, f, v, k, t = 48, 96, 200, 9, torch.bfloat16
    weights = [mat(*s, t, 2 + i, 0, s[1] ** -0.5) for i, s in enumerate(((f, d), (f, d), (v, f), (v, f)))]
    idx, u = lists(n, v, k, t, 5)[1:]
    points = [mat(n, d, t, 20 + i) for i in range(3)]

    def step(x, leaves):
        h = bh.gated_layer(x, leaves[0], leaves[1])
        z = bh.gated_layer(h, leaves[2], leaves[3], "gelu")
        loss = bh.distil_loss(z, idx, u, 0.5)[0].sum()
        return [loss.detach(), *torch.autograd.grad(loss, leaves)]

    wants = [[r.clone() for r in step(x, [w.clone().requires_grad_() for w in weights])] for x in points]
    x, leaves = points[0].clone(), [w.clone().requires_grad_() for w in weights]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(x, leaves)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, leaves)
    for turn in (1, 0, 2, 2):
        x.copy_(points[turn])
        graph.replay()
        torch.cuda.synchronize()
        for i, (p, q) in enumerate(zip(got[1:], wants[turn][1:])):
            assert torch.equal(p, q), (turn, i)
        assert abs(float(got[0]) - float(wants[turn][0])) <= n * 2.0 ** -23 * max(1.0, abs(float(wants[turn][0])))
        step(x, [w.clone().requires_grad_() for w in weights])
