"""Timed cases of the operators that train and serve the heads a cache certifies.

Five kinds of pass, each what a program that learns or serves classification heads runs:

* ortho:    orthogonalise a matrix (or a batch of equal ones) by Newton-Schulz products;
* step:     one optimiser step built on it: momentum, orthogonalised direction, decayed weight;
* forward:  logits of feature rows under a shared head and each row's own low-rank adapter;
* backward: the gradients of that: features and both factors of every adapter;
* loss:     softmax cross entropy of logits, per-row losses and the gradient of the logits.

Plain forms compute in FP32 and round once, to the type of the output.
"""
import math

import torch

own = False

DEV = torch.device("cuda", 0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # a, b, c of X <- aX + (bA + cAA)X, A = XX^T
STEPS, EPS = 5, 1e-7
LR, BETA, DECAY = 0.02, 0.95, 0.01


def listed():
    def ortho(name, dtype, batch, rows, cols):
        return {"name": name, "kind": "ortho", "dtype": dtype, "batch": batch, "rows": rows, "cols": cols}

    def step(name, dtype, batch, rows, cols):
        return {"name": name, "kind": "step", "dtype": dtype, "batch": batch, "rows": rows, "cols": cols}

    def head(name, kind, dtype, tokens, d, classes, adapters, rank, grouped, bias=True):
        return {"name": name, "kind": kind, "dtype": dtype, "tokens": tokens, "d": d, "classes": classes,
                "adapters": adapters, "rank": rank, "grouped": grouped, "bias": bias}

    def loss(name, dtype, tokens, classes):
        return {"name": name, "kind": "loss", "dtype": dtype, "tokens": tokens, "classes": classes}

    return [
        # The head of the Tiny-ImageNet-shaped cache: one small matrix, where launches count.
        ortho("ortho_head", "f32", 1, 200, 256),
        # A tall FP32 projection with odd sides: full precision, transposed iteration.
        ortho("ortho_tall_odd", "f32", 1, 2001, 1003),
        # A training step over both factors of 64 adapters at once: many small wide matrices.
        step("step_adapters", "f32", 64, 16, 1024),
        # A training step of the square projections of a large layer: the tensor cores' case.
        step("step_large", "bf16", 2, 4096, 4096),
        # One feature against the Tiny-ImageNet-shaped head, eight tenants' adapters: the single-token form.
        head("serve_single", "forward", "f32", 1, 256, 200, 8, 8, False),
        # One decoding batch: 48 rows of 64 tenants in no order; the shared weight's bytes bound it.
        head("serve_batch", "forward", "bf16", 48, 4096, 4096, 64, 16, False),
        # Prefill: ragged requests one after another, each with its adapter.
        head("prefill", "forward", "bf16", 8192, 4096, 4096, 16, 16, True),
        # One insert batch of FP32 features (the batch of the timed builds), rows of ten tenants mixed.
        head("insert_batch", "forward", "f32", 65_536, 256, 200, 10, 8, False),
        # Training, BF16: ragged requests, eight adapters of rank 32.
        head("train_bf16", "backward", "bf16", 4096, 2048, 4096, 8, 32, True, False),
        # Training, FP32, odd sizes, rows mixed.
        head("train_odd", "backward", "f32", 4095, 500, 1000, 5, 6, False, False),
        # A vocabulary-sized loss with an odd width.
        loss("loss_wide", "bf16", 4096, 50_001),
        # The scale workload's 200 classes, one insert batch of rows.
        loss("loss_classes", "f32", 65_536, 200),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def side(lo, hi):
        v = log(lo, hi)
        return max(1, v // 64 * 64) if v >= 128 and rng.random() < 0.5 else v

    kind = rng.choice(["ortho", "step", "forward", "forward", "backward", "loss"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "bf16"])}
    if kind in ("ortho", "step"):
        c["rows"], c["cols"] = side(8, 4096), side(8, 4096)
        small = min(c["rows"], c["cols"])
        most = (1 << 32) // max(1, small * c["rows"] * c["cols"] // 8)
        c["batch"] = max(1, min(log(1, 64), most))
    elif kind == "loss":
        c["classes"] = log(2, 50_001)
        c["tokens"] = min(log(1, 65_536), max(1, 200_000_000 // c["classes"]))
    else:
        c["d"], c["classes"] = side(16, 4096), side(10, 4096)
        c["adapters"], c["rank"] = log(1, 64), rng.choice([1, 4, 6, 8, 16, 16, 32, 64])
        c["grouped"], c["bias"] = rng.random() < 0.5, kind == "forward" and rng.random() < 0.7
        most = (1 << 37) // (c["d"] * c["classes"]) if kind == "forward" else (1 << 35) // (c["d"] * c["classes"])
        c["tokens"] = max(1, min(log(1, 65_536), most, 60_000_000 // max(c["classes"], c["adapters"] * c["rank"])))
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 1_000_003 + 11)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _gradient(gen, batch, rows, cols):
    """What an optimiser meets: a few strong directions over noise."""
    k = max(1, min(rows, cols) // 8)
    decay = torch.logspace(0, -2, k, device=DEV)
    strong = torch.matmul(_normal(gen, batch, rows, k) * decay, _normal(gen, batch, k, cols))
    return (strong + 0.5 * _normal(gen, batch, rows, cols)) * 1e-3


def _adapter_ids(gen, case):
    """Each row's adapter: ragged requests in order, or rows of all tenants mixed; one request in ten has none."""
    n, g = case["tokens"], case["adapters"]
    ids = torch.randint(0, g, (n,), generator=gen, device=DEV)
    ids = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.1, torch.full_like(ids, -1), ids)
    if case["grouped"]:
        # requests start where a row is drawn as a start, and take the id drawn there
        start = torch.rand(n, generator=gen, device=DEV) < max(1.0 / n, 0.004)
        at = torch.cummax(torch.where(start, torch.arange(n, device=DEV), torch.zeros_like(ids)), 0).values
        ids = ids[at]
    return ids.to(torch.int32)


def prepare(case, seed):
    gen, dt, kind = _gen(seed), DTYPES[case["dtype"]], case["kind"]
    s = {"kind": kind}
    if kind == "ortho":
        s["x"] = _gradient(gen, case["batch"], case["rows"], case["cols"]).to(dt)
    elif kind == "step":
        b, m, n = case["batch"], case["rows"], case["cols"]
        s["grad"] = _gradient(gen, b, m, n).to(dt)
        s["momentum"] = _gradient(gen, b, m, n)
        s["weight"] = (_normal(gen, b, m, n) / math.sqrt(n)).to(dt)
        s["out"] = (torch.empty_like(s["weight"]), torch.empty_like(s["momentum"]))
    elif kind == "loss":
        n, c = case["tokens"], case["classes"]
        z = 3.0 * _normal(gen, n, c)
        # a row's tenant does not offer every class: those logits are -inf
        z.masked_fill_(torch.rand(1, c, generator=gen, device=DEV) < 0.02, -math.inf)
        y = torch.randint(0, c, (n,), generator=gen, device=DEV)
        z.scatter_(1, y[:, None], 3.0 * _normal(gen, n, 1))
        y = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.05, torch.full_like(y, -1), y)
        s["logits"], s["target"] = z.to(dt), y.to(torch.int32)
        s["weight"] = torch.rand(n, generator=gen, device=DEV) / n
    else:
        n, d, c, g, r = case["tokens"], case["d"], case["classes"], case["adapters"], case["rank"]
        s["x"] = _normal(gen, n, d).to(dt)
        s["W"] = (_normal(gen, c, d) / math.sqrt(d)).to(dt)
        s["bias"] = 0.1 * _normal(gen, c) if case["bias"] else None
        s["A"] = (_normal(gen, g, r, d) / math.sqrt(d)).to(dt)
        s["B"] = (_normal(gen, g, c, r) / math.sqrt(r)).to(dt)
        s["adapter"] = _adapter_ids(gen, case)
        s["scales"] = 0.25 + torch.rand(g, generator=gen, device=DEV)
        if kind == "backward":
            s["dy"] = (_normal(gen, n, c) / n).to(dt)
    return s


# ---------------------------------------------------------------- one pass
def _iterate(x):
    """Newton-Schulz products in FP32 on the matrices in their wide orientation."""
    a, b, c = COEFFICIENTS
    tall = x.shape[-2] > x.shape[-1]
    x = x.transpose(-2, -1) if tall else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(-2, -1))
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.transpose(-2, -1) if tall else x


def _masked(product, adapter, scales, rank):
    """(rows, adapters * rank): the low-rank products of each row's own adapter, times its scale; 0 elsewhere."""
    g = scales.shape[0]
    pick = (adapter[:, None] == torch.arange(g, device=DEV)[None, :]) * scales[None, :]
    return product * pick.repeat_interleave(rank, dim=1)


def run(state):
    kind = state["kind"]
    if own:
        from paper_2608_13144_gb300 import heads

        if kind == "ortho":
            return heads.orthogonalize(state["x"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
        if kind == "step":
            return heads.orthogonal_step(state["weight"], state["grad"], state["momentum"], lr=LR, beta=BETA,
                                         weight_decay=DECAY, steps=STEPS, coefficients=COEFFICIENTS, eps=EPS,
                                         out=state["out"])
        if kind == "loss":
            return heads.cross_entropy(state["logits"], state["target"], state["weight"])
        if kind == "forward":
            return heads.adapted_logits(state["x"], state["W"], state["A"], state["B"], state["adapter"],
                                        bias=state["bias"], scales=state["scales"])
        return heads.adapted_logits_backward(state["dy"], state["x"], state["W"], state["A"], state["B"],
                                             state["adapter"], scales=state["scales"])
    if kind == "ortho":
        return _iterate(state["x"].float()).to(state["x"].dtype)
    if kind == "step":
        grad, dt = state["grad"].float(), state["weight"].dtype
        momentum = BETA * state["momentum"] + (1 - BETA) * grad
        o = _iterate((1 - BETA) * grad + BETA * momentum)
        scale = math.sqrt(max(1.0, o.shape[-2] / o.shape[-1]))
        return ((1 - LR * DECAY) * state["weight"].float() - LR * scale * o).to(dt), momentum
    if kind == "loss":
        z, y, w = state["logits"].float(), state["target"].long(), state["weight"]
        w = torch.where(y >= 0, w, torch.zeros_like(w))
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        at = y.clamp(min=0)[:, None]
        loss = w * (torch.log(total) + top - z.gather(1, at))[:, 0]
        hot = torch.arange(z.shape[1], device=DEV)[None, :] == at
        return loss, (w[:, None] * (e / total - hot.float())).to(state["logits"].dtype)
    dt, adapter, scales = state["x"].dtype, state["adapter"], state["scales"]
    x, W, A, B = (state[k].float() for k in ("x", "W", "A", "B"))
    g, r, d = A.shape
    c = W.shape[0]
    A_all, B_all = A.reshape(g * r, d), B.transpose(1, 2).reshape(g * r, c)
    u = _masked(torch.matmul(x, A_all.t()), adapter, scales, r)
    if kind == "forward":
        y = torch.matmul(x, W.t()) + torch.matmul(u, B_all)
        return (y if state["bias"] is None else y + state["bias"]).to(dt)
    dy = state["dy"].float()
    v = _masked(torch.matmul(dy, B_all.t()), adapter, scales, r)
    dx = torch.matmul(dy, W) + torch.matmul(v, A_all)
    dA = torch.matmul(v.t(), x).reshape(g, r, d)
    dB = torch.matmul(u.t(), dy).reshape(g, r, c).transpose(1, 2)
    return dx.to(dt), dA.to(dt), dB.contiguous().to(dt)


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_polar(x):
    """Each matrix by its Gram matrix's powers: X <- X (aI + bS + cS^2), S = X^T X on the smaller side."""
    a, b, c = COEFFICIENTS
    done = []
    for m in x.double():
        tall = m.shape[0] > m.shape[1]
        y = m if tall else m.t()
        y = y / (torch.linalg.vector_norm(y) + EPS)
        eye = torch.eye(y.shape[1], dtype=torch.float64, device=DEV)
        for _ in range(STEPS):
            s = y.t() @ y
            y = y @ (a * eye + s @ (b * eye + c * s))
        done.append(y if tall else y.t())
    return torch.stack(done)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "ortho":
        return _exact_polar(s["x"])
    if kind == "step":
        g = s["grad"].double()
        m = s["momentum"].double()
        m = m + (g - m) * (1 - BETA)
        o = _exact_polar(g + (m - g) * BETA)
        scale = math.sqrt(max(1.0, case["rows"] / case["cols"]))
        return s["weight"].double() * (1 - LR * DECAY) - o * (LR * scale), m
    if kind == "loss":
        n, c = case["tokens"], case["classes"]
        if n * c > 250_000_000:
            return None
        z = s["logits"].double()
        lp = torch.log_softmax(z, 1)
        y, w = s["target"].long(), s["weight"].double()
        rows = torch.arange(n, device=DEV)[y >= 0]
        loss = torch.zeros(n, dtype=torch.float64, device=DEV)
        loss[rows] = -w[rows] * lp[rows, y[rows]]
        grad = torch.zeros_like(z)
        grad[rows] = lp[rows].exp()
        grad[rows, y[rows]] -= 1.0
        return loss, grad * w[:, None]
    x, W, A, B = (s[k].double() for k in ("x", "W", "A", "B"))
    ids, scales = s["adapter"].long(), s["scales"].double()
    if kind == "forward":
        y = x @ W.t() + (0.0 if s["bias"] is None else s["bias"].double())
        for i in range(case["adapters"]):
            at = (ids == i).nonzero()[:, 0]
            y[at] += scales[i] * ((x[at] @ A[i].t()) @ B[i].t())
        return y
    dy = s["dy"].double()
    dx, dA, dB = dy @ W, torch.zeros_like(A), torch.zeros_like(B)
    for i in range(case["adapters"]):
        at = (ids == i).nonzero()[:, 0]
        v = scales[i] * (dy[at] @ B[i])
        dx[at] += v @ A[i]
        dA[i] = v.t() @ x[at]
        dB[i] = scales[i] * (dy[at].t() @ (x[at] @ A[i].t()))
    return dx, dA, dB


# ---------------------------------------------------------------- work
def work(case):
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind in ("ortho", "step"):
        b, m, n = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # the Gram matrix and its square are symmetric: half of each product
        flops = STEPS * b * (m * m * n + m ** 3 + 2 * m * m * n)
        return {"bytes": b * m * n * (2 * e if kind == "ortho" else 3 * e + 8), "flops": flops}
    if kind == "loss":
        n, c = case["tokens"], case["classes"]
        return {"bytes": 2 * n * c * e + 12 * n, "flops": 5 * n * c}
    n, d, c, r = case["tokens"], case["d"], case["classes"], case["rank"]
    used = min(case["adapters"], n)
    weights = (c * d + used * r * (c + d)) * e
    if kind == "forward":
        return {"bytes": weights + n * (d + c) * e + 4 * n, "flops": 2 * n * (d * c + r * (d + c))}
    return {"bytes": weights + n * (2 * d + c) * e + case["adapters"] * r * (c + d) * e + 4 * n,
            "flops": 2 * n * (d * c + 3 * r * (d + c))}
