"""Measured cases of the operators that train a map from data to its embedding.

A map (an encoder of dense layers, each followed by a layer norm) takes every
point's features to its place in the embedding; the t-SNE gradient at those places
goes back through the layer norms to the weight matrices, whose update is
orthogonalised before it is applied.  The operators are the layer norm's forward
and backward pass over all points, the orthogonalisation of a matrix by
Newton-Schulz products, and the whole momentum step of a weight matrix with it.

    listed(), draw(rng)     the cases, and one more of the same ranges
    prepare(case, seed)     what the program has in hand before the call
    run(state)              one pass
    work(case)              bytes and flops a pass cannot do without
    exact(case, seed)       the same outputs in 64 bits

With `own` false a pass is computed in plain torch operations in 32 bits, rounded
once at the end; with `own` true by this repository's kernels.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS_NORM = 1e-5   # added to a row's variance
EPS_ORTH = 1e-7   # added to a matrix' norm
STEPS = 5
COEF = (3.4445, -4.7750, 2.0315)  # one Newton-Schulz step: a X + (b A + c A^2) X, A = X X^T
LEARNING_RATE, MOMENTUM, DECAY = 0.02, 0.95, 0.01


# ------------------------------------------------------------------ the cases
# op: "norm" and "norm_backward" (n points of d features, `pad` unused features behind
# each row, weights of type `param`), "orthogonalise" and "muon" (batch matrices of
# rows x cols; the second with momentum, decay and the weights' update).
def _norm(name, op, n, d, dtype, param="f32", pad=0):
    return dict(name=name, op=op, n=n, d=d, dtype=dtype, param=param, pad=pad)


def _orth(name, op, rows, cols, dtype, batch=1):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, batch=batch)


def listed():
    return [
        # one new point is placed by a trained map: latency alone
        _norm("norm_1_point", "norm", 1, 512, "bf16", "bf16"),
        # 50 principal components of 1.3M cells, fp16: short rows of odd alignment
        _norm("norm_1300k_50", "norm", 1_300_000, 50, "f16"),
        # a hidden layer of an image data set (70k points), at a width off every tile
        _norm("norm_70k_777", "norm", 70_000, 777, "f32"),
        # the backward pass at the smallest real run, 2000 points
        _norm("norm_back_2k", "norm_backward", 2_000, 128, "f32"),
        # the same layer of 70k points, a slice of a wider buffer
        _norm("norm_back_70k_slice", "norm_backward", 70_001, 500, "bf16", "bf16", pad=12),
        # the largest: the hidden layer of 1.3M points
        _norm("norm_back_1300k", "norm_backward", 1_300_000, 256, "bf16"),
        # the last layer of a small map, hidden to the plane: two rows
        _orth("orth_2x128", "orthogonalise", 2, 128, "f32"),
        # a hidden layer in bf16
        _orth("orth_1024", "orthogonalise", 1024, 1024, "bf16"),
        # the widest layer
        _orth("orth_4096", "orthogonalise", 4096, 4096, "bf16"),
        # the first layer of a map of 50 components
        _orth("muon_256x50", "muon", 256, 50, "f32"),
        # a tall layer of odd sizes in 32 bits
        _orth("muon_1999x777", "muon", 1999, 777, "f32"),
        # eight equal layers at once
        _orth("muon_8x512", "muon", 512, 512, "bf16", batch=8),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "orthogonalise", "muon"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op.startswith("norm"):
        d = _log_uniform(rng, 2, 8192)
        n = _log_uniform(rng, 1, min(1_300_000, 300_000_000 // (d * BYTES[dtype])))
        c = _norm("", op, n, d, dtype, rng.choice(["f32", dtype]), rng.choice([0, 0, rng.randint(1, 64)]))
    else:
        rows, cols = _log_uniform(rng, 1, 2500), _log_uniform(rng, 1, 2500)
        batch = rng.choice([1, 1, rng.randint(2, 8)]) if rows * cols < 1_000_000 else 1
        c = _orth("", op, rows, cols, dtype, batch)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs (plain torch)
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _rows(gen, n, d, pad, dtype, make):
    """An n x d tensor of `make`'s values, the first columns of rows d + pad long."""
    buf = torch.empty((n, d + pad), device=DEV, dtype=dtype)
    if pad:
        buf[:, d:] = float("nan")  # not a feature: nothing may read it
    step = max(1, (1 << 26) // d)
    for i in range(0, n, step):
        buf[i:i + step, :d] = make(min(step, n - i))
    return buf[:, :d]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1_000_003 + 17)
    T = TYPES[case["dtype"]]
    if case["op"].startswith("norm"):
        n, d, pad, TP = case["n"], case["d"], case["pad"], TYPES[case["param"]]
        centre, spread = 0.5 * _randn(gen, d), torch.exp(0.5 * _randn(gen, d))  # features of unequal size
        # a dense layer's outputs: every point has a scale of its own
        x = _rows(gen, n, d, pad, T, lambda m: torch.exp(0.3 * _randn(gen, m, 1)) * (centre + spread * _randn(gen, m, d)))
        s = dict(case=case, x=x, weight=(1.0 + 0.2 * _randn(gen, d)).to(TP), bias=(0.1 * _randn(gen, d)).to(TP))
        if case["op"] == "norm_backward":
            x32 = x.float()
            mean = x32.mean(1)
            s["mean"], s["rstd"] = mean, torch.rsqrt((x32 - mean[:, None]).square().mean(1) + EPS_NORM)
            drift = 0.02 * _randn(gen, d)
            s["dy"] = _rows(gen, n, d, pad, T, lambda m: drift + 0.1 * _randn(gen, m, d))
        return s
    b, r, c = case["batch"], case["rows"], case["cols"]
    k = min(r, c)
    # a layer's gradient, a sum of outer products: a spectrum that falls off, over noise of every direction
    fall = torch.arange(1, k + 1, device=DEV, dtype=torch.float32) ** -0.5
    G = (_randn(gen, b, r, k) * fall) @ _randn(gen, b, k, c) + 0.3 * _randn(gen, b, r, c)
    s = dict(case=case, G=(1e-3 * G).to(T))
    if case["op"] == "muon":
        s["W"] = (_randn(gen, b, r, c) / math.sqrt(c)).to(T)
        s["M"] = 1e-2 * _randn(gen, b, r, c)  # the momentum is kept in 32 bits
    return s


# ------------------------------------------------------------------ one pass
def _plain_norm(x, weight, bias):
    x32 = x.float()
    mean = x32.mean(1)
    centred = x32 - mean[:, None]
    rstd = torch.rsqrt(centred.square().mean(1) + EPS_NORM)
    y = centred * rstd[:, None] * weight.float() + bias.float()
    return y.to(x.dtype), mean, rstd


def _plain_norm_backward(dy, x, weight, mean, rstd):
    dy32 = dy.float()
    xhat = (x.float() - mean[:, None]) * rstd[:, None]
    g = dy32 * weight.float()
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx.to(x.dtype), (dy32 * xhat).sum(0).to(weight.dtype), dy32.sum(0).to(weight.dtype)


def _plain_orthogonal(U):
    """Newton-Schulz steps on a batch of 32-bit matrices, the shorter side first."""
    tall = U.shape[1] > U.shape[2]
    X = U.mT if tall else U
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + EPS_ORTH)
    a, b, c = COEF
    for _ in range(STEPS):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


def _scale(case):
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def _plain_muon(W, G, M, case):
    M.mul_(MOMENTUM).add_(G.float())
    O = _plain_orthogonal(G.float() + MOMENTUM * M)
    W.copy_((1.0 - LEARNING_RATE * DECAY) * W.float() - LEARNING_RATE * _scale(case) * O)


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2212_11506_amd as bh
        if op == "norm":
            return bh.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS_NORM)
        if op == "norm_backward":
            return bh.layer_norm_backward(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"])
        if op == "orthogonalise":
            return bh.orthogonalise(state["G"], steps=STEPS, coefficients=COEF, eps=EPS_ORTH)
        bh.muon_step(state["W"], state["G"], state["M"], LEARNING_RATE, MOMENTUM, nesterov=True, weight_decay=DECAY,
                     scale=_scale(state["case"]), steps=STEPS, coefficients=COEF, eps=EPS_ORTH)
        return state["W"], state["M"]
    if op == "norm":
        return _plain_norm(state["x"], state["weight"], state["bias"])
    if op == "norm_backward":
        return _plain_norm_backward(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"])
    if op == "orthogonalise":
        return _plain_orthogonal(state["G"].float()).to(state["G"].dtype)
    _plain_muon(state["W"], state["G"], state["M"], state["case"])
    return state["W"], state["M"]


# ------------------------------------------------------------------ floors
def work(case):
    e = BYTES[case["dtype"]]
    if case["op"].startswith("norm"):
        n, d, p = case["n"], case["d"], BYTES[case["param"]]
        if case["op"] == "norm":
            return {"bytes": 2 * n * d * e + 8 * n + 2 * d * p, "flops": 8 * n * d}
        return {"bytes": 3 * n * d * e + 8 * n + 3 * d * p, "flops": 14 * n * d}
    b, m, k = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # the symmetric products at half their operations, either on X itself or on X X^T alone
    on_x = STEPS * (3 * m * m * k + m ** 3)
    on_gram = 3 * m * m * k + (4 * STEPS - 3) * m ** 3
    flops = b * min(on_x, on_gram)
    if case["op"] == "orthogonalise":
        return {"bytes": 2 * b * m * k * e, "flops": flops}
    return {"bytes": b * m * k * (3 * e + 8), "flops": flops}


# ------------------------------------------------------------------ 64 bits
def _chunks(n, d):
    step = max(1, (1 << 24) // d)
    return [(i, min(n, i + step)) for i in range(0, n, step)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        n, d = s["x"].shape
        y = torch.empty((n, d), device=DEV, dtype=torch.float64)
        mean, rstd = (torch.empty(n, device=DEV, dtype=torch.float64) for _ in range(2))
        for i, j in _chunks(n, d):
            v, m = torch.var_mean(s["x"][i:j].double(), 1, correction=0)
            mean[i:j], rstd[i:j] = m, (v + EPS_NORM) ** -0.5
            y[i:j] = (s["x"][i:j].double() - m[:, None]) / (v + EPS_NORM).sqrt()[:, None] * s["weight"].double() + s["bias"].double()
        return y, mean, rstd
    if case["op"] == "norm_backward":
        n, d = s["x"].shape
        dx = torch.empty((n, d), device=DEV, dtype=torch.float64)
        dw, db = (torch.zeros(d, device=DEV, dtype=torch.float64) for _ in range(2))
        w = s["weight"].double()
        for i, j in _chunks(n, d):
            dy, x, r = s["dy"][i:j].double(), s["x"][i:j].double(), s["rstd"][i:j].double()
            z = (x - s["mean"][i:j].double()[:, None]) * r[:, None]
            t = dy * w
            dx[i:j] = (r / d)[:, None] * (d * t - t.sum(1)[:, None] - z * (t * z).sum(1)[:, None])
            dw += (dy * z).sum(0)
            db += dy.sum(0)
        return dx, dw, db
    if case["op"] == "orthogonalise":
        return _exact_orthogonal(s["G"].double())
    M = MOMENTUM * s["M"].double() + s["G"].double()
    O = _exact_orthogonal(s["G"].double() + MOMENTUM * M)
    return s["W"].double() * (1.0 - LEARNING_RATE * DECAY) - LEARNING_RATE * _scale(case) * O, M


def _exact_orthogonal(U):
    """All steps are polynomials of A = X X^T that commute: their product Q is formed on the shorter side
    (with A B^2 the next A), then applied to U once."""
    if U.shape[1] > U.shape[2]:
        return _exact_orthogonal(U.mT.contiguous()).mT.contiguous()
    X = U / (torch.linalg.vector_norm(U, dim=(1, 2), keepdim=True) + EPS_ORTH)
    one = torch.eye(U.shape[1], device=DEV, dtype=torch.float64)
    A, Q = X @ X.mT.contiguous(), one
    for _ in range(STEPS):
        B = COEF[0] * one + COEF[1] * A + COEF[2] * (A @ A)
        Q, A = B @ Q, B @ A @ B
    return Q @ X
