"""Timed cases of the operators that answer with heads' probabilities, learn from a teacher's and normalise features.

Five kinds of pass, each what a program that serves or trains classification heads runs:

* score:      log-probability of each row's given class, entropy and most probable classes;
* score_grad: the gradient of those log-probabilities and entropies (a policy's step, an entropy bonus);
* distill:    the divergence of a row's softmax from a teacher's most probable classes, and its gradient;
* norm:       layer norm of feature rows, with the statistics that its gradient needs;
* norm_grad:  its gradients: features, weight and bias.

Plain forms compute in FP32 and round once, to the type of the output.
"""
import math

import torch

own = False

DEV = torch.device("cuda", 0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    def probs(name, kind, dtype, rows, classes, top=0, temperature=1.0):
        return {"name": name, "kind": kind, "dtype": dtype, "rows": rows, "classes": classes, "top": top,
                "temperature": temperature}

    def norm(name, kind, dtype, rows, d):
        return {"name": name, "kind": kind, "dtype": dtype, "rows": rows, "d": d}

    return [
        # One answer of the Tiny-ImageNet-shaped head with its five best classes: launches count.
        probs("score_single", "score", "f32", 1, 200, 5),
        # One token of a vocabulary-sized head, odd width, 20 alternatives: the single-token form of a long row.
        probs("score_token", "score", "bf16", 1, 50_001, 20),
        # A scored prompt: every position of it against its next token.
        probs("score_prompt", "score", "bf16", 4096, 50_001, 20),
        # One insert batch of rows over the scale workload's classes, what a teacher's answers are kept as.
        probs("score_classes", "score", "f32", 65_536, 200, 5, 2.0),
        # A training step on given tokens with an entropy bonus.
        probs("policy_tokens", "score_grad", "bf16", 4096, 50_001),
        # The same over a thousand classes, FP32, odd sizes.
        probs("policy_odd", "score_grad", "f32", 4095, 1001, 0, 0.7),
        # A vocabulary-sized student and a teacher's 64 best tokens of each position.
        probs("distill_tokens", "distill", "bf16", 4096, 50_001, 64, 2.0),
        # A head of the scale workload's classes that learns from a larger model's ten best, one insert batch.
        probs("distill_classes", "distill", "f32", 65_536, 200, 10, 4.0),
        # A decoding batch's features before their head.
        norm("norm_decode", "norm", "bf16", 48, 4096),
        # Prefill: the features of long requests.
        norm("norm_prefill", "norm", "bf16", 16_384, 4096),
        # Training, BF16, wide features.
        norm("norm_train", "norm_grad", "bf16", 16_384, 4096),
        # Training, FP32: one insert batch of the Tiny-ImageNet-shaped features.
        norm("norm_features", "norm_grad", "f32", 65_536, 256),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["score", "score", "score_grad", "distill", "distill", "norm", "norm_grad"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "bf16"])}
    if kind in ("norm", "norm_grad"):
        d = log(8, 16_384)
        c["d"] = max(8, d // 64 * 64) if d >= 128 and rng.random() < 0.5 else d
        c["rows"] = min(log(1, 65_536), (33_000_000 if c["dtype"] == "f32" else 66_000_000) // c["d"])
    else:
        n = log(2, 150_000)
        c["classes"] = max(2, n // 8 * 8) if n >= 64 and rng.random() < 0.5 else n
        c["rows"] = min(log(1, 65_536), (100_000_000 if c["dtype"] == "f32" else 200_000_000) // c["classes"])
        most = min(64 if kind == "distill" else 128, c["classes"] // 2)
        c["top"] = 0 if kind == "score_grad" else log(1, most)
        if kind == "score" and rng.random() < 0.2:
            c["top"] = 0
        c["temperature"] = rng.choice([0.5, 0.7, 1.0, 1.0, 2.0, 4.0])
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 1_000_003 + 29)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV)


def _logits(gen, n, c):
    """Logits of unit-scale noise whose spread differs from row to row, and the classes that are masked (-inf)."""
    z = _normal(gen, n, c) * (1.0 + 3.0 * _uniform(gen, n, 1))
    masked = _uniform(gen, 1, c) < 0.02
    masked[:, :(c + 1) // 2] = False  # half of the classes at least are there for all
    return z, masked


def prepare(case, seed):
    gen, dt, kind = _gen(seed), DTYPES[case["dtype"]], case["kind"]
    s = {"kind": kind}
    if kind in ("norm", "norm_grad"):
        n, d = case["rows"], case["d"]
        # a few features stand out, and rows are not centred
        x = _normal(gen, n, d) * torch.exp(_normal(gen, 1, d)) + 0.5 * _normal(gen, n, 1)
        s["x"] = x.to(dt)
        s["weight"], s["bias"] = 1.0 + 0.2 * _normal(gen, d), 0.1 * _normal(gen, d)
        if kind == "norm_grad":
            s["dy"] = (_normal(gen, n, d) / n).to(dt)
            s["stats"] = _norm_stats(s["x"].float())[1]
        return s
    n, c, k = case["rows"], case["classes"], case["top"]
    z, masked = _logits(gen, n, c)
    s["top"], s["temperature"] = k, case["temperature"]
    if kind == "distill":
        # the teacher agrees with the student by and large; some rows have fewer answers, some none
        best = (0.7 * z + _normal(gen, n, c)).masked_fill_(masked, -math.inf).topk(k, dim=1)
        index = best.indices.to(torch.int32)
        has = torch.where(_uniform(gen, n, 1) < 0.1, (_uniform(gen, n, 1) * (k + 1)).long(), torch.full((n, 1), k, device=DEV))
        s["index"] = torch.where(torch.arange(k, device=DEV)[None, :] < has, index, torch.full_like(index, -1))
        s["teacher"] = best.values
        s["weight"] = _uniform(gen, n) / n
    else:
        y = torch.randint(0, (c + 1) // 2, (n,), generator=gen, device=DEV)
        s["target"] = torch.where(_uniform(gen, n) < 0.05, torch.full_like(y, -1), y).to(torch.int32)
    s["logits"] = z.masked_fill_(masked, -math.inf).to(dt)
    if kind == "score_grad":
        s["norm"] = _softmax_stats(s["logits"].float(), case["temperature"])[0]
        s["dlogprob"] = _normal(gen, n) / n
        s["dentropy"] = -0.01 * _uniform(gen, n) / n
    return s


# ---------------------------------------------------------------- one pass
def _softmax_stats(z, temperature):
    """(norm, t, e): of each row the maximum, the logarithm of sum e, e = exp(t), t = (z - maximum) / temperature, and
    the mean of -t under the softmax."""
    top = z.amax(1, keepdim=True)
    t = (z - top) / temperature
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    mean = (e * torch.where(e > 0, -t, torch.zeros_like(t))).sum(1, keepdim=True) / total
    return torch.cat([top, torch.log(total), mean], 1), t, e


def _best(z, k):
    """Columns of the k largest values of each row in order, the lowest first among equals."""
    bits = (z + 0.0).view(torch.int32)  # (-0 counts as 0)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    order = order * (1 << 32) + (0x7FFFFFFF - torch.arange(z.shape[1], device=DEV))[None, :]
    return 0x7FFFFFFF - (order.topk(k, dim=1).values & 0x7FFFFFFF)


def _norm_stats(x):
    """(centred rows, their mean and 1 / sqrt(variance + eps))."""
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    return xc, torch.cat([mean, torch.rsqrt(xc.square().mean(1, keepdim=True) + EPS)], 1)


def run(state):
    kind = state["kind"]
    if own:
        from paper_2608_13144_gb300 import heads

        if kind == "score":
            r = heads.log_probs(state["logits"], state["target"], top=state["top"], temperature=state["temperature"])
            return (r.logprob, r.entropy, r.norm) + ((r.top, r.index) if state["top"] else ())
        if kind == "score_grad":
            return heads.log_probs_backward(state["logits"], state["norm"], state["target"], state["dlogprob"],
                                            state["dentropy"], temperature=state["temperature"])
        if kind == "distill":
            return heads.distill(state["logits"], state["teacher"], state["index"], state["weight"],
                                 temperature=state["temperature"])
        if kind == "norm":
            return heads.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS)
        return heads.layer_norm_backward(state["dy"], state["x"], state["stats"], state["weight"])
    if kind in ("norm", "norm_grad"):
        x, w, dt = state["x"].float(), state["weight"], state["x"].dtype
        if kind == "norm":
            xc, stats = _norm_stats(x)
            return (xc * stats[:, 1:] * w + state["bias"]).to(dt), stats
        mean, rstd = state["stats"][:, :1], state["stats"][:, 1:]
        dy, xh = state["dy"].float(), (x - mean) * rstd
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return dx.to(dt), (dy * xh).sum(0), dy.sum(0)
    z, dt, temperature = state["logits"].float(), state["logits"].dtype, state["temperature"]
    if kind == "distill":
        v, w = state["teacher"], state["weight"]
        there = state["index"] >= 0
        any_ = there.any(1, keepdim=True)
        v = torch.where(there, v, torch.full_like(v, -math.inf)) / temperature
        v = torch.where(any_, v, torch.zeros_like(v))
        best = v.amax(1, keepdim=True)
        e = torch.exp(v - best)
        log_q = v - best - torch.log(e.sum(1, keepdim=True))
        q = e / e.sum(1, keepdim=True)
        norm, t, e = _softmax_stats(z, temperature)
        at = state["index"].clamp(min=0).long()
        gap = torch.where(q > 0, q * (log_q - (t.gather(1, at) - norm[:, 1:2])), torch.zeros_like(q))
        w = torch.where(any_[:, 0], w, torch.zeros_like(w))
        p = e / e.sum(1, keepdim=True)
        p.scatter_add_(1, at, torch.where(there, -q, torch.zeros_like(q)))
        return w * temperature * temperature * gap.sum(1), (p * (w * temperature)[:, None]).to(dt)
    y = state["target"].long()
    at, valid = y.clamp(min=0)[:, None], y >= 0
    if kind == "score":
        norm, t, e = _softmax_stats(z, temperature)
        logprob = torch.where(valid, t.gather(1, at)[:, 0] - norm[:, 1], torch.zeros_like(norm[:, 1]))
        entropy = norm[:, 1] + norm[:, 2]
        if not state["top"]:
            return logprob, entropy, norm
        index = _best(z, state["top"])
        return logprob, entropy, norm, t.gather(1, index) - norm[:, 1:2], index.to(torch.int32)
    top, log_sum, mean = state["norm"].split(1, 1)
    t = (z - top) / temperature
    p = torch.exp(t - log_sum)
    g_p = torch.where(valid, state["dlogprob"], torch.zeros_like(state["dlogprob"]))[:, None]
    g_h = state["dentropy"][:, None]
    dz = -p * (g_p + g_h * torch.where(p > 0, t + mean, torch.zeros_like(t)))
    dz.scatter_add_(1, at, g_p)
    return (dz / temperature).to(dt)


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("norm", "norm_grad"):
        x, w = s["x"].double(), s["weight"].double()
        if kind == "norm":
            var, mean = torch.var_mean(x, dim=1, keepdim=True, correction=0)
            rstd = (var + EPS) ** -0.5
            return torch.addcmul(s["bias"].double(), (x - mean) * rstd, w), torch.cat([mean, rstd], 1)
        # from the statistics as given: dx = rstd (I - 11'/d - xh xh'/d) (w dy)
        mean, rstd = s["stats"].double()[:, :1], s["stats"].double()[:, 1:]
        x = torch.sub(x, mean).mul_(rstd)
        g = s["dy"].double()
        dw, db = torch.einsum("nd,nd->d", g, x), torch.einsum("nd->d", g)
        g = g * w
        dot = torch.einsum("nd,nd->n", g, x)[:, None] / case["d"]
        return (g - torch.einsum("nd->n", g)[:, None] / case["d"] - x * dot) * rstd, dw, db
    n, c, k, temperature = case["rows"], case["classes"], case["top"], case["temperature"]
    z = s["logits"].double()
    lp = torch.log_softmax(z / temperature, 1)
    rows = torch.arange(n, device=DEV)
    if kind == "distill":
        loss, grad = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros_like(z)
        live = (s["index"] >= 0).any(1).nonzero()[:, 0]
        there, at = s["index"][live] >= 0, s["index"][live].clamp(min=0).long()
        lq = torch.log_softmax(torch.where(there, s["teacher"][live].double() / temperature, -math.inf), 1)
        gap = torch.where(there, lq.exp() * (lq - lp[live].gather(1, at)), 0.0)
        w = s["weight"].double()[live]
        loss[live] = w * temperature ** 2 * gap.sum(1)
        part = lp[live].exp()
        part.scatter_add_(1, at, torch.where(there, -lq.exp(), 0.0))
        grad[live] = part * (w * temperature)[:, None]
        return loss, grad
    y = s["target"].long()
    at = rows[y >= 0]
    p = lp.exp()
    if kind == "score_grad":
        # through the log-probabilities l: dH/dl = -p (l + 1), dz = (v - p sum v) / temperature
        v = torch.where(p > 0, p * (lp + 1.0), 0.0) * -s["dentropy"].double()[:, None]
        v[at, y[at]] += s["dlogprob"].double()[at]
        return (v - p * v.sum(1, keepdim=True)) / temperature
    logprob = torch.zeros(n, dtype=torch.float64, device=DEV)
    logprob[at] = lp[at, y[at]]
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    top = z.amax(1)
    log_sum = torch.logsumexp(z / temperature, 1) - top / temperature
    out = logprob, entropy, torch.stack([top, log_sum, entropy - log_sum], 1)
    if not k:
        return out
    index = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    return out + (lp.gather(1, index), index.to(torch.int32))


# ---------------------------------------------------------------- work
def work(case):
    kind, e, n = case["kind"], 4 if case["dtype"] == "f32" else 2, case["rows"]
    if kind == "norm":
        return {"bytes": 2 * n * case["d"] * e + 8 * case["d"] + 8 * n, "flops": 8 * n * case["d"]}
    if kind == "norm_grad":
        return {"bytes": 3 * n * case["d"] * e + 12 * case["d"] + 8 * n, "flops": 14 * n * case["d"]}
    c, k = case["classes"], case["top"]
    if kind == "score":
        return {"bytes": n * c * e + n * (4 + 4 + 4 + 12 + 8 * k), "flops": 6 * n * c}
    if kind == "score_grad":
        return {"bytes": 2 * n * c * e + n * (4 + 12 + 4 + 4), "flops": 8 * n * c}
    return {"bytes": 2 * n * c * e + n * (8 * k + 4 + 4), "flops": 8 * n * c}
