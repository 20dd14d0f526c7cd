"""The operators that train and serve heads, through the binding, against plain
64-bit forms on the CPU.

Tolerances. An FP32 product sum of K terms on the tensor cores is three FP16
products of operands split in two: each operand is kept to 2^-22 of itself (or
2^-40 of its row's maximum), the product of the two low parts (2^-22) is left
out, and the sum of K terms in FP32 is off by at most K 2^-24 of the terms'
absolute sum (a third of the additions of a K-term loop, each truncated). With
S the absolute sum of all terms of an output element and K the terms along its
longest chain, an element is within (2^-20 + K 2^-24) S of the exact one,
then rounded to its type. BF16 products are exact in FP32, so the same bound
holds for them.

The iteration of orthogonalize amplifies rounding by what its polynomial does
to small singular values, so its tolerance is measured, not fixed: the 64-bit
iteration is run with every product rounded by a random relative error of the
unit that the operator keeps (2^-21 for FP32, 2^-11 for BF16), and the result
may be off by eight times what that changes.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -9}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    return torch.device("cuda", 0)


@pytest.fixture(scope="module")
def heads(dev):
    from paper_2608_13144_gb300 import heads
    yield heads
    assert heads.operator_errors(dev) == 0


def f64(t):
    return t.detach().cpu().double()


def within(got, want, tol, what=""):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    ok = ~(nan | inf)
    off = (got - want).abs()[ok] - tol.expand_as(want)[ok]
    assert off.numel() == 0 or off.max() <= 0, (what, float(off.max()), int((off > 0).sum()), off.numel())


# ---------------------------------------------------------------- adapters
def adapted_case(dev, dtype, n, d, c, g, r, ids, seed=0, scales=True, spread=1.0):
    gen = torch.Generator().manual_seed(1000 * seed + n + 7 * d + c)
    def rnd(*s):
        return torch.randn(*s, generator=gen)
    x, W = rnd(n, d), rnd(c, d) / math.sqrt(d)
    A, B = rnd(g, r, d) / math.sqrt(d), rnd(g, c, r) / math.sqrt(r)
    dy = rnd(n, c)
    if spread != 1.0:  # rows of very different sizes
        x *= torch.exp2(torch.randint(-20, 20, (n, 1), generator=gen).float())
        W *= torch.exp2(torch.randint(-12, 12, (c, 1), generator=gen).float())
        dy *= torch.exp2(torch.randint(-20, 20, (n, 1), generator=gen).float())
    if ids == "mixed":
        a = torch.randint(-1, g + 1, (n,), generator=gen)  # -1 and g: none
    elif ids == "grouped":
        a = torch.sort(torch.randint(-1, g, (n,), generator=gen)).values
    elif ids == "one":
        a = torch.full((n,), g - 1)
    else:
        a = torch.full((n,), -1)
    s = 0.25 + torch.rand(g, generator=gen) if scales else None
    bias = rnd(c)
    t = dict(x=x.to(dtype), W=W.to(dtype), A=A.to(dtype), B=B.to(dtype), dy=dy.to(dtype))
    t = {k: v.to(dev) for k, v in t.items()}
    return t, a.to(torch.int32).to(dev), None if s is None else s.to(dev), bias.to(dev)


def adapted_exact(t, ids, scales, bias):
    """(y, dx, dA, dB) and for each the absolute sum of its terms."""
    x, W, A, B, dy = (f64(t[k]) for k in ("x", "W", "A", "B", "dy"))
    g, r, d = A.shape
    s = torch.ones(g, dtype=torch.float64) if scales is None else f64(scales)
    ids = ids.cpu().long()
    out = []
    for f in (lambda v: v, torch.abs):
        x_, W_, A_, B_, dy_ = f(x), f(W), f(A), f(B), f(dy)
        y = x_ @ W_.t() + (0 if bias is None else f(f64(bias)))
        dx, dA, dB = dy_ @ W_, torch.zeros_like(A), torch.zeros_like(B)
        for i in range(g):
            at = (ids == i).nonzero()[:, 0]
            if not len(at):
                continue
            u, v = s[i] * (x_[at] @ A_[i].t()), s[i] * (dy_[at] @ B_[i])
            y[at] += u @ B_[i].t()
            dx[at] += v @ A_[i]
            dA[i], dB[i] = v.t() @ x_[at], dy_[at].t() @ u
        out.append((y, dx, dA, dB))
    return out


def tolerance(dtype, want, terms, K):
    return 2 * UNIT[dtype] * want.abs() + (2.0 ** -20 + K * 2.0 ** -24) * terms + 1e-37


SHAPES = [
    # n, d, c, g, r, ids
    (1, 1, 1, 1, 1, "one"), (1, 256, 200, 8, 8, "mixed"), (1, 64, 10, 3, 4, "none"), (2, 33, 7, 2, 3, "mixed"),
    (5, 500, 129, 4, 6, "mixed"), (16, 1024, 300, 7, 16, "mixed"), (17, 130, 513, 64, 16, "mixed"),
    (48, 520, 264, 64, 16, "mixed"), (64, 128, 128, 1, 128, "one"), (65, 72, 1000, 5, 1, "mixed"),
    (127, 264, 72, 3, 32, "grouped"), (128, 512, 256, 4, 16, "none"), (129, 96, 257, 9, 24, "mixed"),
    (300, 248, 520, 16, 8, "grouped"), (700, 320, 384, 40, 64, "mixed"), (1500, 136, 200, 3, 100, "grouped"),
    (2049, 64, 96, 2, 8, "grouped"), (3000, 256, 10, 300, 8, "mixed"), (4097, 48, 72, 10, 5, "mixed"),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_adapted(dev, heads, dtype, shape):
    n, d, c, g, r, ids = shape
    t, a, s, bias = adapted_case(dev, dtype, n, d, c, g, r, ids)
    (y, dx, dA, dB), (ty, tdx, tdA, tdB) = adapted_exact(t, a, s, bias)
    got = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s)
    assert got.dtype == dtype
    within(got, y, tolerance(dtype, y, ty, d + r), "y")
    gx, gA, gB = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)
    within(gx, dx, tolerance(dtype, dx, tdx, c + r), "dx")
    within(gA, dA, tolerance(dtype, dA, tdA, c + n), "dA")
    within(gB, dB, tolerance(dtype, dB, tdB, d + n), "dB")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 40, 400])
def test_adapted_rows_of_all_sizes(dev, heads, dtype, n):
    """Rows of x, W and dy whose sizes differ by up to 2^40: each output
    element keeps its precision relative to its own terms."""
    t, a, s, bias = adapted_case(dev, dtype, n, 200, 136, 3, 8, "mixed", seed=3, spread=2.0)
    (y, dx, dA, dB), (ty, tdx, tdA, tdB) = adapted_exact(t, a, s, None)
    got = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, scales=s)
    within(got, y, tolerance(dtype, y, ty, 208), "y")
    gx, gA, gB = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)
    within(gx, dx, tolerance(dtype, dx, tdx, 144), "dx")
    within(gA, dA, tolerance(dtype, dA, tdA, 136 + n), "dA")
    within(gB, dB, tolerance(dtype, dB, tdB, 200 + n), "dB")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 33, 500])
def test_adapted_strides_and_offsets(dev, heads, dtype, n):
    """Rows of wider matrices, bases off the 16-byte boundaries, an output
    with a row stride: nothing beside the rows is read into a result or
    written."""
    d, c = 120, 152
    t, a, s, bias = adapted_case(dev, dtype, n, d, c, 4, 8, "mixed", seed=5)
    (y, dx, dA, dB), (ty, tdx, tdA, tdB) = adapted_exact(t, a, s, bias)

    def inside(m, left, right):
        w = torch.full((m.shape[0], left + m.shape[1] + right), math.nan, dtype=dtype, device=dev)
        w[:, left:left + m.shape[1]] = m
        return w[:, left:left + m.shape[1]]

    for left, right in ((1, 2), (3, 0), (8, 8), (0, 1)):
        x, W, dy = inside(t["x"], left, right), inside(t["W"], right, left), inside(t["dy"], left, 5)
        wide = torch.full((n, left + c + right), 7.0, dtype=dtype, device=dev)
        got = heads.adapted_logits(x, W, t["A"], t["B"], a, bias=bias, scales=s, out=wide[:, left:left + c])
        within(got, y, tolerance(dtype, y, ty, d + 8), "y")
        assert bool((wide[:, :left] == 7).all()) and bool((wide[:, left + c:] == 7).all())
        gx, gA, gB = heads.adapted_logits_backward(dy, x, W, t["A"], t["B"], a, scales=s)
        within(gx, dx, tolerance(dtype, dx, tdx, c + 8), "dx")
        within(gA, dA, tolerance(dtype, dA, tdA, c + n), "dA")
        within(gB, dB, tolerance(dtype, dB, tdB, d + n), "dB")


def test_adapted_without_adapters_or_rows(dev, heads):
    for dtype in (F32, BF16):
        x, W = torch.randn(9, 40, device=dev).to(dtype), torch.randn(24, 40, device=dev).to(dtype)
        A, B = x.new_empty(0, 1, 40), x.new_empty(0, 24, 1)
        ids = torch.zeros(9, dtype=torch.int32, device=dev)
        want = f64(x) @ f64(W).t()
        terms = f64(x).abs() @ f64(W).abs().t()
        within(heads.adapted_logits(x, W, A, B, ids), want, tolerance(dtype, want, terms, 40))
        dx, dA, dB = heads.adapted_logits_backward(want.to(dtype).to(dev), x, W, A, B, ids)
        assert dA.shape == A.shape and dB.shape == B.shape and dx.shape == x.shape
        A, B = torch.randn(2, 3, 40, device=dev).to(dtype), torch.randn(2, 24, 3, device=dev).to(dtype)
        none = ids[:0]
        assert heads.adapted_logits(x[:0], W, A, B, none).shape == (0, 24)
        dx, dA, dB = heads.adapted_logits_backward(x.new_empty(0, 24), x[:0], W, A, B, none)
        assert dx.shape == (0, 40) and not dA.any() and not dB.any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 30, 260])
def test_adapted_non_finite_rows_stay_apart(dev, heads, dtype, n):
    """A NaN or an infinity in one row of x or of an adapter reaches the
    outputs of that row or adapter, and no other."""
    t, a, s, _ = adapted_case(dev, dtype, n + 3, 136, 88, 3, 8, "mixed", seed=9)
    a[:3] = torch.tensor([0, 1, -1], dtype=torch.int32)
    a[3:] = torch.where(a[3:] == 2, torch.ones_like(a[3:]), a[3:])
    clean = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, scales=s)
    x, A = t["x"].clone(), t["A"].clone()
    x[0, 5], x[2, 7] = math.nan, math.inf
    A[2] = math.nan  # no row uses it
    got = heads.adapted_logits(x, t["W"], A, t["B"], a, scales=s)
    assert torch.isnan(got[0]).all()
    assert not torch.isfinite(got[2]).any()
    keep = torch.ones(n + 3, dtype=torch.bool, device=dev)
    keep[0] = keep[2] = False
    assert torch.equal(got[keep], clean[keep])


def test_adapted_repeats_bit_for_bit(dev, heads):
    for dtype in (F32, BF16):
        t, a, s, bias = adapted_case(dev, dtype, 1111, 200, 312, 6, 12, "mixed", seed=2)
        one = [heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s),
               *heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)]
        for _ in range(3):
            two = [heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s),
                   *heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)]
            assert all(torch.equal(p, q) for p, q in zip(one, two))


def test_adapted_order_of_rows_does_not_matter(dev, heads):
    """A row's logits depend on the row and its adapter alone."""
    for dtype in (F32, BF16):
        t, a, s, bias = adapted_case(dev, dtype, 640, 256, 192, 5, 16, "mixed", seed=4)
        y = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s)
        at = torch.argsort(a, stable=True)
        z = heads.adapted_logits(t["x"][at], t["W"], t["A"], t["B"], a[at], bias=bias, scales=s)
        tol = 2 * UNIT[dtype] * f64(y).abs() + 2 ** -12
        within(z, f64(y)[at.cpu()], tol[at.cpu()])


@pytest.mark.parametrize("n", [1, 20, 300])
def test_adapted_gradient_against_differences(dev, heads, n):
    """sum(dy * y) is linear in each of x, A and B alone, so the difference of
    two FP32 forward passes gives each gradient's product with a direction."""
    t, a, s, _ = adapted_case(dev, F32, n, 72, 40, 3, 4, "mixed", seed=6)
    grads = dict(zip(("x", "A", "B"), heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a,
                                                                     scales=s)))
    for name, g in grads.items():
        gen = torch.Generator(device=dev).manual_seed(3)
        step = torch.randn(t[name].shape, generator=gen, device=dev)
        val = []
        for sign in (1.0, -1.0):
            q = dict(t)
            q[name] = t[name] + sign * step
            val.append(f64(heads.adapted_logits(q["x"], q["W"], q["A"], q["B"], a, scales=s)))
        diff = float(((val[0] - val[1]) / 2 * f64(t["dy"])).sum())
        # each forward value is within 2^-17 of its size here; n * 40 of them, signs mixed
        size = float((torch.maximum(val[0].abs(), val[1].abs()) * f64(t["dy"]).abs()).sum())
        assert abs(diff - float((f64(g) * f64(step)).sum())) <= 2.0 ** -17 * size + 1e-6, name


def test_adapted_on_another_stream_and_in_a_graph(dev, heads):
    t, a, s, bias = adapted_case(dev, BF16, 200, 256, 192, 5, 16, "mixed", seed=8)
    want = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        got = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s)
    side.synchronize()
    assert torch.equal(got, want)
    x, out = t["x"].clone(), torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        heads.adapted_logits(x, t["W"], t["A"], t["B"], a, bias=bias, scales=s, out=out)
    x.copy_(t["x"].flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, heads.adapted_logits(x, t["W"], t["A"], t["B"], a, bias=bias, scales=s))


# ---------------------------------------------------------------- cross entropy
def loss_exact(z, y, w):
    z, w = f64(z), torch.ones(len(y), dtype=torch.float64) if w is None else f64(w)
    n, c = z.shape
    loss, grad = torch.zeros(n, dtype=torch.float64), torch.zeros(n, c, dtype=torch.float64)
    size = torch.zeros(n, dtype=torch.float64)
    for i, t in enumerate(y.tolist()):
        if not 0 <= t < c:
            continue
        row = z[i]
        if torch.isnan(row).any() or (row == math.inf).any():
            loss[i], grad[i] = math.nan, math.nan
            continue
        top = row.max()
        if top == -math.inf:
            loss[i] = math.inf if w[i] != 0 else 0.0
            continue
        e = torch.exp(row - top)
        p = e / e.sum()
        loss[i] = 0.0 if w[i] == 0 else w[i] * (torch.log(e.sum()) + top - row[t])
        if row[t] == -math.inf:
            loss[i] = math.inf if w[i] != 0 else 0.0
        p[t] -= 1.0
        grad[i] = w[i] * p
        size[i] = w[i].abs() * (top.abs() + (0 if torch.isinf(row[t]) else row[t].abs()) + math.log(c) + 1)
    return loss, grad, size


def check_loss(heads, z, y, w, dtype, **kw):
    loss, grad, size = loss_exact(z, y, w)
    z0 = z.clone()
    got, dz = heads.cross_entropy(z, y, w, **kw)
    assert got.dtype == F32 and dz.dtype == dtype
    # exp to 2^-21 (its argument's rounding times the largest x e^-x included), the sum's c terms
    # in trees and short runs: within 2^-18 of the probabilities; one rounding
    within(got, loss, 2.0 ** -20 * size + 1e-37, "loss")
    wide = (torch.ones(len(y)) if w is None else w.cpu()).double().abs()[:, None]
    within(dz, grad, UNIT[dtype] * 2 * grad.abs() + 2.0 ** -18 * (grad.abs() + wide * 2.0 ** -6) * 1.0 + 1e-37, "grad")
    if not kw.get("in_place"):
        assert torch.equal(torch.nan_to_num(z), torch.nan_to_num(z0))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,c", [(1, 1), (1, 2), (3, 10), (7, 33), (64, 200), (5, 1000), (130, 1023), (9, 4096),
                                 (4, 8193), (3, 20_000), (2, 50_001), (1, 200_003), (1000, 17)])
def test_cross_entropy(dev, heads, dtype, n, c):
    gen = torch.Generator().manual_seed(n * 131 + c)
    z = (4 * torch.randn(n, c, generator=gen)).to(dtype).to(dev)
    y = torch.randint(0, c, (n,), generator=gen).to(torch.int32)
    if n > 2:
        y[1], y[2] = -1, c
    w = torch.rand(n, generator=gen)
    for weight in (None, w.to(dev)):
        check_loss(heads, z, y.to(dev), weight, dtype)
    only, none = heads.cross_entropy(z, y.to(dev), None, need_grad=False)
    assert none is None and torch.equal(only, heads.cross_entropy(z, y.to(dev))[0])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [3, 40, 300, 5000, 30_001])
def test_cross_entropy_masks_and_extremes(dev, heads, dtype, c):
    inf, nan = math.inf, math.nan
    low = float(torch.finfo(dtype).min)
    gen = torch.Generator().manual_seed(c)
    z = torch.randn(14, c, generator=gen)
    y = torch.zeros(14, dtype=torch.int32)
    z[0, 1:] = -inf                     # the target alone
    z[1] = -inf                         # nothing left
    z[2, 0] = -inf                      # a masked target
    z[3, 1:] = low                      # masks of the type's lowest value
    z[4] = low                          # a row of them: uniform
    z[5, c - 1] = inf
    z[6, c // 2] = nan
    z[7, 0] = nan
    y[8], z[8] = -1, nan                # ignored, whatever it holds
    y[9], z[9, 1] = c + 5, inf
    z[10] = 1e4 * z[10]
    z[11] = 3e38 if dtype == F32 else 3e38  # equal, near the largest
    z[12, :c - 1] = -inf                # the mask leaves the last class
    y[12] = c - 1
    z[13] *= 1e-30
    z, y = z.to(dtype).to(dev), y.to(dev)
    check_loss(heads, z, y, None, dtype)
    w = torch.ones(14, device=dev)
    w[:3] = 0
    check_loss(heads, z, y, w, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [10, 130, 4097, 20_001])
def test_cross_entropy_strides_and_in_place(dev, heads, dtype, c):
    gen = torch.Generator().manual_seed(c)
    n = 6
    y = torch.randint(0, c, (n,), generator=gen).to(torch.int32).to(dev)
    for left, right in ((1, 1), (0, 3), (8, 8)):
        wide = torch.full((n, left + c + right), 5.0, dtype=dtype, device=dev)
        wide[:, left:left + c] = torch.randn(n, c, generator=gen).to(dtype).to(dev)
        z = wide[:, left:left + c]
        check_loss(heads, z, y, None, dtype)
        loss, dz = heads.cross_entropy(z.clone(), y)
        loss2, dz2 = heads.cross_entropy(z, y, in_place=True)
        assert dz2 is z and torch.equal(loss, loss2) and torch.equal(dz, dz2)
        assert bool((wide[:, :left] == 5).all()) and bool((wide[:, left + c:] == 5).all())


def test_cross_entropy_gradient_against_differences(dev, heads):
    """Central differences of the FP32 loss with h = 2^-5: off by h^2 / 6
    times the third derivative (below 0.1) and by the loss's rounding over h."""
    gen = torch.Generator().manual_seed(1)
    z = torch.randn(1, 6, generator=gen).to(dev)
    y = torch.tensor([2], dtype=torch.int32, device=dev)
    g = f64(heads.cross_entropy(z, y)[1])[0]
    h = 2.0 ** -5
    for j in range(6):
        e = torch.zeros_like(z)
        e[0, j] = h
        up, dn = (float(heads.cross_entropy(z + s * e, y)[0][0]) for s in (1, -1))
        assert abs((up - dn) / (2 * h) - float(g[j])) <= h * h / 6 * 0.1 + 2.0 ** -19 / h


# ---------------------------------------------------------------- orthogonalise
QUINTIC, POLAR, CUBIC = (3.4445, -4.7750, 2.0315), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)


def ortho_exact(g, steps, coef, eps, unit=0.0, seed=0):
    """64-bit iteration of one matrix; with `unit`, every product is rounded by a random relative error of it."""
    gen = torch.Generator().manual_seed(seed)

    def rounded(v):
        return v if not unit else v * (1 + unit * (2 * torch.rand(v.shape, generator=gen, dtype=torch.float64) - 1))

    x = g if g.shape[0] <= g.shape[1] else g.t()
    x = rounded(x / (torch.linalg.vector_norm(x) + eps))
    for i in range(steps):
        a, b, c = coef[i] if hasattr(coef[0], "__len__") else coef
        s = rounded(x @ x.t())
        x = rounded(a * x + rounded(rounded(b * s + c * (s @ s)) @ x))
    return x if g.shape[0] <= g.shape[1] else x.t()


def check_ortho(heads, got, g, dtype, steps, coef, eps=1e-7):
    want = ortho_exact(g, steps, coef, eps)
    noise = max(float(torch.linalg.vector_norm(ortho_exact(g, steps, coef, eps, 2.0 ** (-21 if dtype == F32 else -11), k)
                                               - want)) for k in range(3))
    off = float(torch.linalg.vector_norm(f64(got) - want))
    size = float(torch.linalg.vector_norm(want))
    assert off <= 8 * noise + 2 * UNIT[dtype] * size, (off, noise, size)
    return want


def matrix(gen, m, n, kind):
    if kind == "normal":
        return torch.randn(m, n, generator=gen)
    k = max(1, min(m, n) // 6)
    strong = torch.randn(m, k, generator=gen) * torch.logspace(0, -2, k) @ torch.randn(k, n, generator=gen)
    return (strong + 0.3 * torch.randn(m, n, generator=gen)) * 1e-3


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 37), (37, 1), (2, 3), (8, 8), (10, 64), (64, 10), (16, 1024), (1000, 24),
                                 (33, 65), (128, 128), (200, 256), (129, 257), (300, 140), (512, 640), (777, 333),
                                 (1030, 1027)])
def test_orthogonalize(dev, heads, dtype, m, n):
    gen = torch.Generator().manual_seed(m * 7 + n)
    for kind, coef, steps in (("strong", QUINTIC, 5), ("normal", POLAR, 7 if m * n < 40_000 else 3)):
        g = matrix(gen, m, n, kind).to(dtype)
        got = heads.orthogonalize(g.to(dev), steps=steps, coefficients=coef)
        assert got.dtype == dtype and got.shape == g.shape
        check_ortho(heads, got, g.double(), dtype, steps, coef)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,m,n", [(3, 16, 200), (5, 130, 70), (2, 260, 300), (40, 8, 64), (7, 1, 9)])
def test_orthogonalize_batches(dev, heads, dtype, batch, m, n):
    gen = torch.Generator().manual_seed(batch)
    g = torch.stack([matrix(gen, m, n, "strong") * 10.0 ** (i - 2) for i in range(batch)]).to(dtype)
    schedule = [QUINTIC, QUINTIC, POLAR, CUBIC]
    got = heads.orthogonalize(g.to(dev), steps=4, coefficients=schedule)
    for i in range(batch):
        check_ortho(heads, got[i], g[i].double(), dtype, 4, schedule)
    one = heads.orthogonalize(g[1].to(dev), steps=4, coefficients=schedule)
    check_ortho(heads, one, g[1].double(), dtype, 4, schedule)


def test_orthogonalize_to_convergence(dev, heads):
    """Enough steps of the polynomial with p(1) = 1, p'(1) = 0 leave
    orthonormal rows, and a head of spectral norm 1 (its unit the FP32 one)."""
    from paper_2608_13144_gb300.lipcache import LipCache
    gen = torch.Generator().manual_seed(0)
    g = torch.randn(100, 128, generator=gen).to(dev)
    o = heads.orthogonalize(g, steps=16, coefficients=POLAR)
    gram = f64(o) @ f64(o).t()
    assert float((gram - torch.eye(100, dtype=torch.float64)).abs().max()) <= 2.0 ** -17
    with LipCache(128, 100, 16, device=dev) as cache:
        assert abs(cache.set_head(o, torch.zeros(100, device=dev)) - 1.0) <= 2.0 ** -17


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(12, 40), (150, 90), (300, 320)])
def test_orthogonalize_extremes(dev, heads, dtype, m, n):
    """Zero, tiny, huge, single-entry and rank-one matrices, and a NaN or an
    infinity that stays in its matrix of the batch."""
    gen = torch.Generator().manual_seed(5)
    base = torch.randn(m, n, generator=gen)
    g = torch.stack([torch.zeros(m, n), base * 1e-12, base * 1e15, torch.zeros(m, n),
                     torch.outer(base[:, 0], base[0]), base, base, base])
    g[3, m // 2, n // 3] = 0.02
    g[5, 1, 2], g[6, 0, 0] = math.nan, math.inf
    g = g.to(dtype)
    got = heads.orthogonalize(g.to(dev))
    assert not got[0].any()
    for i in (1, 2, 3, 4, 7):
        check_ortho(heads, got[i], g[i].double(), dtype, 5, QUINTIC)
    assert torch.isnan(got[5]).all() and torch.isnan(got[6]).all()


def test_orthogonalize_strides_in_place_and_streams(dev, heads):
    gen = torch.Generator().manual_seed(2)
    for dtype in (F32, BF16):
        for left, right in ((0, 3), (1, 0), (8, 8)):
            wide = torch.full((2, 90, left + 130 + right), math.nan, dtype=dtype, device=dev)
            wide[:, :, left:left + 130] = torch.randn(2, 90, 130, generator=gen).to(dtype).to(dev)
            g = wide[:, :, left:left + 130]
            got = heads.orthogonalize(g)
            for i in range(2):
                check_ortho(heads, got[i], f64(g[i]), dtype, 5, QUINTIC)
            dense = g.contiguous()
            side = torch.cuda.Stream(dev)
            side.wait_stream(torch.cuda.current_stream(dev))
            with torch.cuda.stream(side):
                again = heads.orthogonalize(dense, out=dense)
            side.synchronize()
            assert again is dense and torch.equal(dense, got)
            across = torch.randn(130, 90, generator=gen).to(dtype).to(dev).t()  # columns dense, not rows
            check_ortho(heads, heads.orthogonalize(across), f64(across), dtype, 5, QUINTIC)


@pytest.mark.parametrize("wt,gt", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)],
                         ids=["f32", "bf16", "f32_bf16", "bf16_f32"])
@pytest.mark.parametrize("shape", [(16, 256), (3, 200, 64), (260, 300), (1, 1)], ids=str)
@pytest.mark.parametrize("nesterov", [True, False])
def test_orthogonal_step(dev, heads, wt, gt, shape, nesterov):
    gen = torch.Generator().manual_seed(sum(shape))
    b, m, n = (1, *shape) if len(shape) == 2 else shape
    grad = torch.stack([matrix(gen, m, n, "strong") for _ in range(b)]).reshape(shape).to(gt)
    mom = torch.stack([matrix(gen, m, n, "strong") for _ in range(b)]).reshape(shape)
    w = (torch.randn(shape, generator=gen) / math.sqrt(n)).to(wt)
    lr, beta, decay = 0.3, 0.9, 0.1
    g64, m64 = grad.double(), mom.double()
    new = beta * m64 + (1 - beta) * g64
    d = beta * new + (1 - beta) * g64 if nesterov else new
    W, G, M = w.to(dev), grad.to(dev), mom.to(dev)
    ow, om = heads.orthogonal_step(W, G, M, lr, beta, nesterov, decay, out=(torch.empty_like(W), torch.empty_like(M)))
    assert torch.equal(W.cpu(), w) and torch.equal(M.cpu(), mom)
    within(om, new, 4 * UNIT[F32] * (m64.abs() + g64.abs()))
    keep, rate = 1 - lr * decay, lr * math.sqrt(max(1.0, m / n))
    for i in range(b):
        di, wi, oi = (v.reshape(b, m, n)[i] for v in (d, w.double(), ow))
        unit = 2.0 ** (-21 if wt == F32 else -11)
        o = ortho_exact(di, 5, QUINTIC, 1e-7)
        noise = max(float(torch.linalg.vector_norm(ortho_exact(di, 5, QUINTIC, 1e-7, unit, k) - o)) for k in range(3))
        want = keep * wi - rate * o
        off = float(torch.linalg.vector_norm(f64(oi) - want))
        # the direction itself is formed in FP32, an error of the same kind as `noise` measures
        assert off <= 8 * rate * noise + 2 * UNIT[wt] * float(torch.linalg.vector_norm(want)) + 1e-6 * rate
    rw, rm = heads.orthogonal_step(W, G, M, lr, beta, nesterov, decay)
    assert rw is W and rm is M and torch.equal(W, ow) and torch.equal(M, om)


# ---------------------------------------------------------------- refusals
def test_refusals(dev, heads):
    from paper_2608_13144_gb300 import LipCacheError
    x, W = torch.randn(4, 16, device=dev), torch.randn(8, 16, device=dev)
    A, B = torch.randn(2, 3, 16, device=dev), torch.randn(2, 8, 3, device=dev)
    ids = torch.zeros(4, dtype=torch.int32, device=dev)
    ok = dict(x=x, W=W, A=A, B=B, adapter=ids)
    for bad in (dict(x=x.cpu()), dict(x=x.double()), dict(W=W.bfloat16()), dict(W=W[:, :8]), dict(A=A[:, :, :8]),
                dict(B=B[:1]), dict(adapter=ids.long()), dict(adapter=ids[:2]), dict(x=x[0]), dict(bias=W[:, 0][:3]),
                dict(bias=W[:, 0].bfloat16()), dict(scales=x[0]), dict(out=x), dict(out=torch.empty(8, 4, device=dev).t())):
        with pytest.raises(ValueError):
            heads.adapted_logits(**{**ok, **bad})
    with pytest.raises(ValueError):
        heads.adapted_logits_backward(x, x, W, A, B, ids)
    with pytest.raises(LipCacheError) as e:
        heads.adapted_logits(x, W, x.new_zeros(2, 129, 16), x.new_zeros(2, 8, 129), ids)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        heads.cross_entropy(x, ids.long())
    with pytest.raises(ValueError):
        heads.cross_entropy(x.half(), ids)
    with pytest.raises(ValueError):
        heads.cross_entropy(x, ids, ids)
    with pytest.raises(ValueError):
        heads.cross_entropy(x.t(), torch.zeros(16, dtype=torch.int32, device=dev), in_place=True)
    for kw in (dict(coefficients=(1.0, 2.0)), dict(coefficients=[QUINTIC] * 3, steps=4)):
        with pytest.raises(ValueError):
            heads.orthogonalize(x, **kw)
    for kw in (dict(steps=0), dict(steps=33), dict(eps=0.0), dict(coefficients=(math.nan, 0, 0)),
               dict(coefficients=(100.0, 0, 0))):
        with pytest.raises(LipCacheError) as e:
            heads.orthogonalize(x, **kw)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        heads.orthogonalize(x[0])
    with pytest.raises(ValueError):
        heads.orthogonal_step(x, x, x.bfloat16(), 0.1)
    with pytest.raises(ValueError):
        heads.orthogonal_step(x.t(), x.t(), x.t(), 0.1)
    with pytest.raises(LipCacheError):
        heads.orthogonal_step(x, x, x.clone(), 0.1, beta=1.5)
