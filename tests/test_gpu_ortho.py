"""Orthogonalisation by Newton-Schulz products, and the momentum step with it, against the formulas in 64 bits.

Tolerances, as the 2-norm of the difference over that of the result.  An error E before a step is at most a E
after it (a = 3.4445: no divided difference of s (a + b s^2 + c s^4) exceeds it), so errors made at each of five
steps grow to at most a^5 / (a - 1) = 200 times one step's.  fp32 and fp16 outputs: a step's three products of
22-bit operands with fp32 sums are off by about 2^-21 of their size, in random directions: 200 * 2^-21 = 1e-4.
bf16 outputs: B X alone has operands of 11 bits; their errors, 2^-12 in random directions, appear where B X does,
not in a X, and largely at the last steps: 8 * 2^-12 = 2e-3.  Then the output's own rounding, half a unit at most."""
import pytest
import torch

import paper_2212_11506_amd as bh

pytestmark = pytest.mark.gpu
DEV = "cuda"
COEF = (3.4445, -4.7750, 2.0315)
TYPES = [torch.float32, torch.float16, torch.bfloat16]
TOL = {torch.float32: 1e-4, torch.float16: 1e-4 + 2.0 ** -11, torch.bfloat16: 2e-3 + 2.0 ** -8}


def say(*a):
    print(*a, flush=True)


def plain(G, steps=5, coef=COEF, eps=1e-7):
    """The formulas as they stand, in 64 bits on the CPU; coef: one triple or one for each step."""
    G = G.double().cpu()
    if G.dim() == 3:
        return torch.stack([plain(g, steps, coef, eps) for g in G])
    tall = G.shape[0] > G.shape[1]
    X = G.t() if tall else G
    X = X / (X.norm() + eps)
    for k in range(steps):
        a, b, c = coef[k] if hasattr(coef[0], "__len__") else coef
        A = X @ X.t()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.t() if tall else X


def rel(got, want):
    got = got.double().cpu()
    assert got.shape == want.shape
    return float((got - want).norm() / want.norm())


def gauss(*shape, seed=0, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=g)).to(dtype).to(DEV)


# one value, vectors, the two-row last layer, ends inside a tile on either side, squares, both orientations
SHAPES = [(1, 1), (1, 7), (9, 1), (1, 300), (2, 128), (128, 2), (3, 5), (16, 16), (17, 33), (50, 256), (63, 64), (64, 64), (65, 63),
          (64, 1000), (130, 70), (100, 127), (128, 128), (129, 385), (200, 333), (333, 200), (256, 256), (512, 512), (700, 500),
          (1000, 1030)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    say(f"[orth] {shape} {dtype}")
    G = gauss(*shape, seed=shape[0] * 1000 + shape[1], dtype=dtype, scale=1e-2)
    O = bh.orthogonalise(G)
    assert O.dtype == dtype
    assert rel(O, plain(G)) <= TOL[dtype]


def plain_there(G, steps=5, eps=1e-7):
    """plain() of one matrix on the GPU: 64-bit products are the library's."""
    tall = G.shape[0] > G.shape[1]
    X = (G.t() if tall else G).double().contiguous()
    X = X / (X.norm() + eps)
    a, b, c = COEF
    for _ in range(steps):
        A = X @ X.t().contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return (X.t() if tall else X).cpu()


# large enough for each of the larger tiles, with ends inside them
@pytest.mark.parametrize("shape,dtype", [((1999, 777), torch.float32), ((777, 1999), torch.float16), ((2100, 2048), torch.float32),
                                         ((1300, 2500), torch.bfloat16), ((2500, 2200), torch.bfloat16),
                                         ((3000, 2900), torch.float32), ((4000, 4160), torch.bfloat16), ((900, 6000), torch.bfloat16)])
def test_large(shape, dtype):
    say(f"[orth] {shape} {dtype}")
    G = gauss(*shape, seed=11, dtype=dtype)
    r = rel(bh.orthogonalise(G), plain_there(G))
    say(f"[orth] {r:.2e}")
    assert r <= TOL[dtype]


# few directions: X in one block up to its LDS, then cut into slices, few and many; one value over each end
NARROW = [(1, 2048), (16, 2049), (16, 4096), (17, 512), (17, 513), (48, 256), (49, 128), (49, 129), (4200, 64), (64, 256), (64, 257), (32, 512), (32, 513), (33, 256), (257, 64), (5, 1000), (1500, 40), (33, 2048), (33, 2049), (64, 5000),
          (9000, 20), (1, 65536)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", NARROW)
def test_few_directions(shape, dtype):
    say(f"[orth] {shape} {dtype}")
    G = gauss(2, *shape, seed=shape[0] + shape[1], dtype=dtype, scale=1e-3)
    O, want = bh.orthogonalise(G), plain(G)
    assert max(rel(O[k], want[k]) for k in range(2)) <= TOL[dtype]


@pytest.mark.parametrize("dtype", TYPES)
def test_spectra(dtype):
    """Singular values that fall off by 1e4, and eight large ones over noise: errors against the largest would show."""
    g = torch.Generator().manual_seed(5)
    m, n = 192, 320
    fall = torch.randn(m, m, generator=g) @ torch.diag(torch.logspace(0, -4, m)) @ torch.randn(m, n, generator=g)
    spikes = torch.randn(m, 8, generator=g) @ torch.randn(8, n, generator=g) + 0.01 * torch.randn(m, n, generator=g)
    for name, G in (("fall", fall), ("spikes", spikes)):
        G = G.to(dtype).to(DEV)
        r = rel(bh.orthogonalise(G), plain(G))
        say(f"[orth] {name} {dtype} {r:.2e}")
        assert r <= TOL[dtype]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1e8, 1e30])
def test_scale_of_the_input(scale, dtype):
    G = gauss(70, 90, seed=3, scale=1.0).to(torch.float32)
    G = (G * scale).to(dtype)
    # eps is added to the norm: at 1e-30 the formula's result is small too
    for eps in (0.0, 1e-7):
        want = plain(G, eps=eps)
        assert rel(bh.orthogonalise(G, eps=eps), want) <= TOL[dtype] or float(want.abs().max()) < 1e-18


@pytest.mark.parametrize("steps,coef", [(1, COEF), (2, COEF), (8, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0)),
                                        (3, [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)])])
def test_steps_and_coefficients(steps, coef):
    G = gauss(90, 140, seed=4)
    assert rel(bh.orthogonalise(G, steps=steps, coefficients=coef), plain(G, steps, coef)) <= 1e-4


@pytest.mark.parametrize("dtype", TYPES)
def test_the_result_is_nearly_orthogonal(dtype):
    """Singular values come out between 0.65 and 1.25, where those of the input were above a hundredth of its norm."""
    G = gauss(96, 400, seed=6, dtype=dtype)
    s = torch.linalg.svdvals(bh.orthogonalise(G).double().cpu())
    assert float(s.min()) > 0.6 and float(s.max()) < 1.3


@pytest.mark.parametrize("shape", [(40, 60), (60, 40), (200, 150)])
def test_batches_strides_and_in_place(shape):
    r, c = shape
    buf = torch.full((3, r + 2, c + 5), float("nan"), device=DEV)
    G = buf[:, :r, :c]
    G.copy_(gauss(3, r, c, seed=7))
    want = plain(G)
    out = torch.full((3, r, c + 3), 42.0, device=DEV)
    O = bh.orthogonalise(G, out=out[:, :, :c])
    assert max(rel(O[k], want[k]) for k in range(3)) <= 1e-4
    assert bool((out[:, :, c:] == 42.0).all())
    alone = [bh.orthogonalise(G[k].contiguous()) for k in range(3)]
    assert all(torch.equal(O[k], alone[k]) for k in range(3))
    assert bh.orthogonalise(G, out=G) is G and all(torch.equal(G[k], alone[k]) for k in range(3))
    assert bool(torch.isnan(buf[:, r:]).all()) and bool(torch.isnan(buf[:, :, c:]).all())
    same = alone[0].expand(2, r, c)  # one matrix stands for two
    twice = bh.orthogonalise(same)
    assert torch.equal(twice[0], twice[1])
    assert bh.orthogonalise(torch.empty((0, r, c), device=DEV)).shape == (0, r, c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(24, 40), (64, 1000), (96, 136), (400, 304)])
def test_starts_off_every_alignment(shape, dtype):
    G = gauss(*shape, seed=12, dtype=dtype)
    shift = lambda t: torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(t.shape)  # noqa: E731
    W, M = gauss(*shape, seed=13, dtype=dtype, scale=0.1), gauss(*shape, seed=14)
    want = W.clone(), M.clone()
    assert torch.equal(bh.orthogonalise(shift(G), out=shift(torch.zeros_like(G))), bh.orthogonalise(G))
    bh.muon_step(want[0], G, want[1], 0.1)
    W, M = shift(W), shift(M)
    bh.muon_step(W, shift(G), M, 0.1)
    assert torch.equal(W, want[0]) and torch.equal(M, want[1])


@pytest.mark.parametrize("shape", [(8, 8), (20, 300), (300, 200)])
def test_zero_and_nonfinite_matrices(shape):
    G = torch.zeros((3, *shape), device=DEV)
    G[1] = gauss(*shape, seed=8)
    G[2] = gauss(*shape, seed=9)
    G[2, 3, 4] = float("nan")
    O = bh.orthogonalise(G)
    assert bool((O[0] == 0).all()) and bool(torch.isnan(O[2]).all())
    assert rel(O[1], plain(G[1])) <= 1e-4
    G[2, 3, 4] = float("inf")
    assert bool(torch.isnan(bh.orthogonalise(G)[2]).all())
    # the workspace that held NaN serves the next call
    ws = torch.empty(bh.orthogonalise_workspace_size(1, *shape), dtype=torch.uint8, device=DEV)
    bh.orthogonalise(G[2], workspace=ws)
    assert torch.equal(bh.orthogonalise(G[1], workspace=ws), O[1])


def muon64(W, G, M, lr, mu, nesterov, wd, scale):
    W, G, M = (t.double().cpu() for t in (W, G, M))
    M = mu * M + G
    return (1 - lr * wd) * W - lr * scale * plain(G + mu * M if nesterov else M), M


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(2, 64), (64, 50), (300, 130), (3, 96, 96), (2, 256, 70)])
def test_muon_step(shape, nesterov, dtype):
    say(f"[muon] {shape} {dtype} nesterov={nesterov}")
    W, G, M = gauss(*shape, seed=1, dtype=dtype, scale=0.1), gauss(*shape, seed=2, dtype=dtype), gauss(*shape, seed=3)
    lr, mu, wd, scale = 0.5, 0.9, 0.1, 1.25  # a rate that makes the update as large as the weights
    Ww, Mw = muon64(W, G, M, lr, mu, nesterov, wd, scale)
    step = Ww - (1 - lr * wd) * W.double().cpu()
    bh.muon_step(W, G, M, lr, mu, nesterov=nesterov, weight_decay=wd, scale=scale)
    assert float((M.double().cpu() - Mw).abs().max()) <= 4 * 2.0 ** -24 * float(Mw.abs().max() + G.abs().max())
    half = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    err = float((W.double().cpu() - Ww).norm())
    assert err <= TOL[dtype] * float(step.norm()) + 4 * half * float(Ww.norm())


@pytest.mark.parametrize("shape,dtype", [((1000, 1024), torch.bfloat16), ((1500, 700), torch.float16), ((2048, 2100), torch.float32),
                                         ((2300, 2048), torch.bfloat16), ((3000, 2900), torch.float16), ((4000, 4160), torch.bfloat16)])
def test_muon_step_large(shape, dtype):
    """The weights' update by every larger tile, against 64-bit products: the step's own error, and the weights' rounding."""
    W, G, M = gauss(*shape, seed=1, dtype=dtype, scale=0.1), gauss(*shape, seed=2, dtype=dtype), gauss(*shape, seed=3)
    lr, mu, wd, scale = 0.5, 0.9, 0.1, 1.25
    Mw = mu * M.double() + G.double()
    step = plain_there(G.double() + mu * Mw).to(DEV)
    want = (1 - lr * wd) * W.double() - lr * scale * step
    bh.muon_step(W, G, M, lr, mu, nesterov=True, weight_decay=wd, scale=scale)
    assert float((M.double() - Mw).abs().max()) <= 4 * 2.0 ** -24 * float(Mw.abs().max() + G.double().abs().max())
    half = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    err = float((W.double() - want).norm())
    assert err <= TOL[dtype] * lr * scale * float(step.norm()) + 4 * half * float(want.norm())


@pytest.mark.parametrize("shape,dtype", [((101, 77), torch.float32), ((65, 131), torch.bfloat16), ((67, 33), torch.float16)])
def test_muon_step_batch_without_gaps(shape, dtype):
    """Matrices that follow one another, of an odd number of values: each starts at another alignment."""
    W, G, M = gauss(3, *shape, seed=1, dtype=dtype, scale=0.1), gauss(3, *shape, seed=2, dtype=dtype), gauss(3, *shape, seed=3)
    mu = 0.9
    scale = max(1.0, shape[0] / shape[1]) ** 0.5  # where none is given
    Mw = mu * M.double() + G.double()
    steps = [scale * plain_there(G[k].double() + mu * Mw[k]).to(DEV) for k in range(3)]
    want = [W[k].double() - 0.5 * steps[k] for k in range(3)]
    bh.muon_step(W, G, M, 0.5, mu, nesterov=True)
    assert float((M.double() - Mw).abs().max()) <= 4 * 2.0 ** -24 * float(Mw.abs().max() + G.double().abs().max())
    half = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    for k in range(3):
        err = float((W[k].double() - want[k]).norm())
        assert err <= TOL[dtype] * 0.5 * float(steps[k].norm()) + 4 * half * float(want[k].norm())


def test_muon_steps_in_a_graph_and_on_another_stream():
    shape = (192, 130)
    W0, G, M0 = gauss(*shape, seed=1, scale=0.1), gauss(*shape, seed=2), gauss(*shape, seed=3)
    ws = torch.empty(bh.orthogonalise_workspace_size(1, *shape), dtype=torch.uint8, device=DEV)
    W, M, eager = W0.clone(), M0.clone(), []
    for _ in range(3):
        bh.muon_step(W, G, M, 0.1, workspace=ws)
        eager.append((W.clone(), M.clone()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    W, M = W0.clone(), M0.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bh.muon_step(W, G, M, 0.1, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(W, eager[0][0]) and torch.equal(M, eager[0][1])
    W, M = W0.clone(), M0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bh.muon_step(W, G, M, 0.1, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(W, W0), "capture must not run the step"
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(W, eager[k][0]) and torch.equal(M, eager[k][1])
        bh.orthogonalise(W, workspace=ws)  # eager work on the same workspace
        torch.cuda.synchronize()


def test_refusals():
    G = gauss(8, 9)
    for call in (lambda: bh.orthogonalise(G.double()), lambda: bh.orthogonalise(G.t()), lambda: bh.orthogonalise(G, out=G.half()),
                 lambda: bh.orthogonalise(G, out=gauss(9, 9)), lambda: bh.orthogonalise(G, coefficients=(1.0, 2.0)),
                 lambda: bh.muon_step(G, G, G.half(), 0.1), lambda: bh.muon_step(G, G.half(), G, 0.1),
                 lambda: bh.muon_step(G, G, gauss(9, 8), 0.1), lambda: bh.muon_step(G, G[0], G, 0.1)):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: bh.orthogonalise(G, steps=0), bh.BHTSNE_EINVAL),
                         (lambda: bh.orthogonalise(G, coefficients=(100.0, 0.0, 0.0)), bh.BHTSNE_EINVAL),
                         (lambda: bh.orthogonalise(G, eps=-1.0), bh.BHTSNE_EINVAL),
                         (lambda: bh.orthogonalise(G.expand(2, 8, 9), out=gauss(1, 8, 9).expand(2, 8, 9)), bh.BHTSNE_EINVAL),
                         (lambda: bh.muon_step(G, G.clone(), G.clone(), -0.1), bh.BHTSNE_EINVAL),
                         (lambda: bh.orthogonalise(G, workspace=torch.empty(8, dtype=torch.uint8, device=DEV)),
                          bh.BHTSNE_EWORKSPACE)):
        with pytest.raises(bh.BhtsneError) as e:
            call()
        assert e.value.status == status
