"""Measured cases of more operators of a trained map: its hidden layers, a loss from neighbour lists, its 8-bit form.

A map from features to places has gated hidden layers, h = act(x gate^T) (x up^T), and
their backward pass.  A head over classes or landmark points can be trained from
neighbour lists alone: the similarities of a point's k neighbours are a teacher's
largest logits, and the loss is the divergence of the head's softmax from theirs.  A
trained map places many points by products of 8-bit integers, with a scale for each
point and each output.

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


# ------------------------------------------------------------------ the cases
# op: "gated" (n points of d features to f; `keep`: with what the backward pass takes) and
# "gated_backward"; "linear8" (n points of d features to f, in 8 bits); "distil" and
# "distil_backward" (n rows of v logits, k listed neighbours, temperature).  `pad` values lie
# unused behind each row of the points.
def _gated(name, op, n, d, f, dtype, act="silu", keep=False, pad=0):
    return dict(name=name, op=op, n=n, d=d, f=f, dtype=dtype, act=act, keep=keep, pad=pad)


def _linear(name, n, d, f, dtype, bias=True, pad=0):
    return dict(name=name, op="linear8", n=n, d=d, f=f, dtype=dtype, bias=bias, pad=pad)


def _distil(name, op, n, v, k, dtype, temperature=1.0, pad=0):
    return dict(name=name, op=op, n=n, v=v, k=k, dtype=dtype, temperature=temperature, pad=pad)


def listed():
    return [
        # one new point is placed by a trained map: latency, and one read of the weights
        _gated("gated_1_point", "gated", 1, 512, 2048, "bf16"),
        # the first layer on 50 principal components of 1.3M cells: short rows of odd alignment, bound by what is written
        _gated("gated_1300k_50", "gated", 1_300_000, 50, 200, "f16", "gelu"),
        # the largest layer, in training
        _gated("gated_16k", "gated", 16_384, 2048, 8192, "bf16", keep=True),
        # the backward pass at the smallest real run, 2000 points, in 32 bits
        _gated("gated_back_2k", "gated_backward", 2_000, 128, 512, "f32"),
        # widths off every tile, points that are a slice of a wider buffer
        _gated("gated_back_5k_odd", "gated_backward", 5_003, 777, 1999, "f16", "gelu", pad=3),
        # the hidden layer of an image data set (70k points)
        _gated("gated_back_70k", "gated_backward", 70_000, 512, 2048, "bf16"),
        # one new point through a wide 8-bit layer: one read of the weights
        _linear("place_1_point", 1, 2048, 8192, "bf16"),
        # 70k points placed at once
        _linear("place_70k", 70_001, 2000, 2000, "bf16"),
        # 2000 points that are each other's classes, 90 neighbours (perplexity 30), in 32 bits
        _distil("distil_2k", "distil", 2_000, 2_000, 90, "f32"),
        # a batch against all of 70k points
        _distil("distil_70k", "distil", 4_096, 70_001, 90, "bf16"),
        # the backward pass of a smaller batch against as many
        _distil("distil_back_70k", "distil_backward", 2_048, 70_000, 90, "bf16", 2.0),
        # a few points against 1.3M: rows longer than a CU holds
        _distil("distil_back_1300k", "distil_backward", 16, 1_300_000, 30, "f16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["gated", "gated_backward", "linear8", "distil", "distil_backward"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    pad = rng.choice([0, 0, rng.randint(1, 64)])
    if op.startswith("distil"):
        v = _log_uniform(rng, 2, 1_300_000)
        n = _log_uniform(rng, 1, min(100_000, 200_000_000 // v))
        k = _log_uniform(rng, 1, min(v, 256))
        c = _distil("", op, n, v, k, dtype, rng.choice([1.0, 1.0, 0.5, 2.0, 4.0]), pad)
    else:
        d, f = _log_uniform(rng, 2, 4096), _log_uniform(rng, 2, 8192)
        most = 100_000_000_000 if dtype == "f32" and op != "linear8" else 400_000_000_000
        n = _log_uniform(rng, 1, max(1, min(1_300_000, 200_000_000 // max(d, f), most // (4 * d * f))))
        if op == "linear8":
            c = _linear("", n, d, f, dtype, rng.choice([True, False]), pad)
        else:
            c = _gated("", op, n, d, f, dtype, rng.choice(["silu", "gelu"]), rng.choice([True, False]) and op == "gated", pad)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs (plain torch)
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _rows(n, d, pad, dtype, make):
    """An n x d tensor of `make`'s values, the first columns of rows d + pad long."""
    buf = torch.empty((n, d + pad), device=DEV, dtype=dtype)
    if pad:
        buf[:, d:] = float("nan")  # not a value: nothing may read it
    step = max(1, (1 << 26) // d)
    for i in range(0, n, step):
        buf[i:i + step, :d] = make(i, min(n, i + step))
    return buf[:, :d]


def _chunks(n, width):
    step = max(1, (1 << 25) // width)
    return [(i, min(n, i + step)) for i in range(0, n, step)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1_000_003 + 29)
    T, n, pad = TYPES[case["dtype"]], case["n"], case["pad"]
    if case["op"].startswith("distil"):
        v, k, temperature = case["v"], case["k"], case["temperature"]
        # k different points a row, in no order; some lists are shorter (index -1), one row in 50 has no list at all
        idx = torch.randint(1, v // k + 1, (n, k), generator=gen, device=DEV).cumsum(1) - 1
        idx = idx[:, torch.randperm(k, generator=gen, device=DEV)]
        # the nearest first: -d^2 / (2 sigma^2)
        near = -(4.0 * torch.rand((n, k), generator=gen, device=DEV)).square().sort(1).values * temperature
        logits = _rows(n, v, pad, T, lambda i, j: temperature * (1.5 * _randn(gen, j - i, v) - 2.0))
        far = max(1, (1 << 25) // k)
        for i in range(0, n, far):  # a head that has learnt some of it
            part = logits[i:i + far]
            rows = torch.arange(part.shape[0], device=DEV)[:, None]
            part[rows, idx[i:i + far]] = (near[i:i + far] + temperature * (4.0 + _randn(gen, part.shape[0], k))).to(T)
        count = torch.randint(1, k + 1, (n, 1), generator=gen, device=DEV)
        count = torch.where(torch.rand((n, 1), generator=gen, device=DEV) < 0.75, k, count)
        count = torch.where(torch.rand((n, 1), generator=gen, device=DEV) < 0.02, 0, count)
        idx = torch.where(torch.arange(k, device=DEV) < count, idx, -1).to(torch.int32)
        s = dict(case=case, logits=logits, idx=idx, teacher=near)
        if case["op"] == "distil_backward":
            lse = torch.empty(n, device=DEV, dtype=torch.float32)
            for i, j in _chunks(n, v):
                lse[i:j] = torch.logsumexp(logits[i:j].double() / temperature, 1)
            s["lse"], s["dloss"] = lse, 0.5 + torch.rand(n, generator=gen, device=DEV)
        return s
    d, f = case["d"], case["f"]
    spread = torch.exp(0.5 * _randn(gen, d))  # features of unequal size
    x = _rows(n, d, pad, T, lambda i, j: spread * _randn(gen, j - i, d))
    if case["op"] == "linear8":
        w = _randn(gen, f, d) * torch.exp(0.3 * _randn(gen, f, 1)) / math.sqrt(d)
        scale = w.abs().amax(1) / 127.0
        q = (w.double() / scale.double()[:, None]).round().to(torch.int8)
        return dict(case=case, x=x, w=q, w_scale=scale, bias=0.1 * _randn(gen, f) if case["bias"] else None)
    gate, up = ((_randn(gen, f, d) / math.sqrt(d)).to(T) for _ in range(2))
    s = dict(case=case, x=x, gate=gate, up=up)
    if case["op"] == "gated_backward":
        s["a"], s["b"] = (torch.empty((n, f), device=DEV, dtype=T) for _ in range(2))
        for i, j in _chunks(n, f):
            s["a"][i:j] = x[i:j].float() @ gate.float().T
            s["b"][i:j] = x[i:j].float() @ up.float().T
        drift = 0.02 * _randn(gen, f)
        s["dh"] = _rows(n, f, 0, T, lambda i, j: drift + 0.1 * _randn(gen, j - i, f))
    return s


# ------------------------------------------------------------------ one pass
def _act(a, kind):
    """The activation and its derivative, 32 bits."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return a * s, s * (1.0 + a * (1.0 - s))
    phi = 0.5 * torch.erfc(a * -math.sqrt(0.5))
    return a * phi, phi + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_gated(x, gate, up, kind, keep):
    a, b = x.float() @ gate.float().T, x.float() @ up.float().T
    h = (_act(a, kind)[0] * b).to(x.dtype)
    return (h, a.to(x.dtype), b.to(x.dtype)) if keep else h


def _plain_gated_backward(dh, x, gate, up, a, b, kind):
    value, slope = _act(a.float(), kind)
    da, db = dh.float() * b.float() * slope, dh.float() * value
    dx = da @ gate.float() + db @ up.float()
    x32 = x.float()
    return dx.to(x.dtype), (da.T @ x32).to(gate.dtype), (db.T @ x32).to(up.dtype)


def _plain_linear8(x, w, w_scale, bias):
    x32 = x.float()
    scale = x32.abs().amax(1, keepdim=True) / 127.0
    # a value next to the border of two integers: in 64 bits; a row of zeros stays zero
    q = (x32.double() / torch.where(scale > 0, scale, 1.0).double()).round().float()
    out = (q @ w.float().T) * scale * w_scale
    return (out if bias is None else out + bias).to(x.dtype)


def _teacher(idx, teacher, temperature):
    """The listed neighbours' probabilities and their logarithms (0 and 0 where there is none)."""
    there = idx >= 0
    u = torch.where(there, teacher.float() / temperature, -math.inf)
    top = u.amax(1, keepdim=True)
    e = torch.exp(u - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(1, keepdim=True)
    t = torch.where(there, e / total, 0.0)
    return t, torch.where(t > 0, u - top - total.log(), 0.0)


def _plain_distil(logits, idx, teacher, temperature):
    z = logits.float() / temperature
    top = z.amax(1)
    lse = top + (z - top[:, None]).exp().sum(1).log()
    t, log_t = _teacher(idx, teacher, temperature)
    log_q = z.gather(1, idx.clamp(min=0).long()) - lse[:, None]
    return torch.where(t > 0, t * (log_t - log_q), 0.0).sum(1), lse


def _plain_distil_backward(dloss, logits, idx, teacher, lse, temperature):
    t = _teacher(idx, teacher, temperature)[0]
    factor = dloss[:, None] / temperature
    dz = factor * (logits.float() / temperature - lse[:, None]).exp() * (idx >= 0).any(1, keepdim=True)
    return dz.scatter_add_(1, idx.clamp(min=0).long(), -factor * t).to(logits.dtype)


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2212_11506_amd as bh
        if op == "gated":
            return bh.gated_layer(state["x"], state["gate"], state["up"], case["act"], keep=case["keep"])
        if op == "gated_backward":
            return bh.gated_layer_backward(state["dh"], state["x"], state["gate"], state["up"], state["a"], state["b"], case["act"])
        if op == "linear8":
            return bh.linear_i8(state["x"], state["w"], state["w_scale"], bias=state["bias"])
        if op == "distil":
            return bh.distil_loss(state["logits"], state["idx"], state["teacher"], case["temperature"])
        return bh.distil_loss_backward(state["dloss"], state["logits"], state["idx"], state["teacher"], state["lse"],
                                       case["temperature"])
    if op == "gated":
        return _plain_gated(state["x"], state["gate"], state["up"], case["act"], case["keep"])
    if op == "gated_backward":
        return _plain_gated_backward(state["dh"], state["x"], state["gate"], state["up"], state["a"], state["b"], case["act"])
    if op == "linear8":
        return _plain_linear8(state["x"], state["w"], state["w_scale"], state["bias"])
    if op == "distil":
        return _plain_distil(state["logits"], state["idx"], state["teacher"], case["temperature"])
    return _plain_distil_backward(state["dloss"], state["logits"], state["idx"], state["teacher"], state["lse"], case["temperature"])


# ------------------------------------------------------------------ floors
def work(case):
    e, n = BYTES[case["dtype"]], case["n"]
    if case["op"].startswith("distil"):
        v, lists = case["v"], 8 * n * case["k"]
        if case["op"] == "distil":
            return {"bytes": n * v * e + lists + 8 * n, "flops": 4 * n * v}
        return {"bytes": 2 * n * v * e + lists + 8 * n, "flops": 4 * n * v}
    d, f = case["d"], case["f"]
    if case["op"] == "linear8":
        return {"bytes": n * d * e + f * d + n * f * e + 4 * f * (2 if case["bias"] else 1), "flops": 2 * n * d * f}
    if case["op"] == "gated":
        return {"bytes": (n * d + 2 * d * f + n * f * (3 if case["keep"] else 1)) * e, "flops": 4 * n * d * f}
    return {"bytes": (2 * n * d + 3 * n * f + 4 * d * f) * e, "flops": 8 * n * d * f}


# ------------------------------------------------------------------ 64 bits
def _exact_gate(a, kind):
    if kind == "silu":
        s = torch.sigmoid(a)
        return a * s, s + a * s * torch.sigmoid(-a)
    phi = torch.special.ndtr(a)
    return a * phi, phi + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("distil"):
        return _exact_distil(case, s)
    x, n, f = s["x"], case["n"], case["f"]
    if case["op"] == "linear8":
        out = torch.empty((n, f), device=DEV, dtype=torch.float64)
        w = s["w"].double().T.contiguous()
        for i, j in _chunks(n, max(f, case["d"])):
            top = x[i:j].abs().amax(1).float()
            step = (top / 127).double()  # the scale is a 32-bit number
            q = torch.where(step[:, None] > 0, torch.round(x[i:j].double() / step[:, None]), 0.0)
            out[i:j] = (q @ w) * (step[:, None] * s["w_scale"].double())
            if s["bias"] is not None:
                out[i:j] += s["bias"].double()
        return out
    gate, up, kind = s["gate"].double(), s["up"].double(), case["act"]
    if case["op"] == "gated":
        h, a, b = (torch.empty((n, f), device=DEV, dtype=torch.float64) for _ in range(3))
        for i, j in _chunks(n, f):
            a[i:j], b[i:j] = x[i:j].double() @ gate.T, x[i:j].double() @ up.T
            h[i:j] = _exact_gate(a[i:j], kind)[0] * b[i:j]
        return (h, a, b) if case["keep"] else h
    dx = torch.empty(x.shape, device=DEV, dtype=torch.float64)
    dgate, dup = torch.zeros_like(gate), torch.zeros_like(up)
    for i, j in _chunks(n, max(f, case["d"])):
        value, slope = _exact_gate(s["a"][i:j].double(), kind)
        dh, points = s["dh"][i:j].double(), x[i:j].double()
        da, db = dh * s["b"][i:j].double() * slope, dh * value
        dx[i:j] = torch.addmm(da @ gate, db, up)
        dgate += da.T @ points
        dup += db.T @ points
    return dx, dgate, dup


def _exact_distil(case, s):
    n, v, temperature = case["n"], case["v"], case["temperature"]
    loss, lse = (torch.empty(n, device=DEV, dtype=torch.float64) for _ in range(2))
    dz = torch.empty((n, v), device=DEV, dtype=torch.float64) if case["op"] == "distil_backward" else None
    for i, j in _chunks(n, v):
        z = s["logits"][i:j].double() / temperature
        listed_ = s["idx"][i:j] >= 0
        u = (s["teacher"][i:j].double() / temperature).masked_fill(~listed_, -math.inf)
        log_t = torch.log_softmax(u, 1).masked_fill(~listed_, 0.0)  # a row without a list is all masked
        t = log_t.exp() * listed_
        at = s["idx"][i:j].long() * listed_
        if dz is None:
            lse[i:j] = torch.logsumexp(z, 1)
            loss[i:j] = (t * (log_t - z.gather(1, at) + lse[i:j, None])).sum(1)
        else:
            g = s["dloss"][i:j].double()[:, None] / temperature
            dz[i:j] = g * torch.exp(z - s["lse"][i:j].double()[:, None]) * t.sum(1, keepdim=True)
            dz[i:j].scatter_add_(1, at, -g * t)
    return (loss, lse) if dz is None else dz
