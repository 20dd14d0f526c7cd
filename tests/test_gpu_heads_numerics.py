"""Precision, ranges and refusals of the operators that train and serve heads:
numbers far from one, non-finite values and their neighbours, what a caller is
told. Same 64-bit forms as test_gpu_heads.py; tolerances are derived at each
test.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_heads import (  # noqa: E402,F401
    BF16, F32, POLAR, QUINTIC, UNIT, adapted_case, adapted_exact, check_ortho, dev, f64, heads, ortho_exact,
    tolerance, within)


# ---------------------------------------------------------------- the loss's precision
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [2, 33, 200, 5000, 50_001])
@pytest.mark.parametrize("offset", [0.0, 20.0, 1000.0, 10_000.0, -10_000.0])
def test_cross_entropy_of_confident_rows(dev, heads, dtype, c, offset):
    """The loss keeps its own precision wherever the logits stand. Logits are at most 30 below the
    largest: each exponential is off by 30 2^-22 at most (its argument's three roundings) and the
    sum by 2^-18, as in check_loss; 2^-16 of the loss covers both and the logarithm."""
    gen = torch.Generator().manual_seed(c)
    n = 24
    z = -14.0 - 16.0 * torch.rand(n, c, generator=gen)
    y = torch.randint(0, c, (n,), generator=gen).to(torch.int32)
    rows = torch.arange(n)
    z[rows, y.long()] = torch.linspace(-30.0, 0.0, n)  # targets that lose, tie and win
    z[: n // 2, c // 2] = torch.linspace(-30.0, 0.0, n // 2)
    z[-4:] -= 14.0 * (torch.arange(c)[None, :] != y[-4:, None].long())  # almost certain
    z[-4:].clamp_(min=-30.0)
    z = (z + offset).to(dtype).to(dev)
    # the others' sum over the target's term, so that 64 bits hold the sure rows too
    e = torch.exp(f64(z) - f64(z)[rows, y.long()][:, None])
    e[rows, y.long()] = 0.0
    others = e.sum(1)
    want, grad = torch.log1p(others), e / (1 + others)[:, None]
    grad[rows, y.long()] = -others / (1 + others)
    got, dz = heads.cross_entropy(z, y.to(dev))
    within(got, want, 2.0 ** -16 * want.abs() + 1e-37, "loss")
    within(dz, grad, 2 * UNIT[dtype] * grad.abs() + 2.0 ** -16 * grad.abs() + 1e-37, "grad")


# ---------------------------------------------------------------- beta near one
@pytest.mark.parametrize("shape", [(16, 200), (90, 130), (90, 128), (3, 70, 65)], ids=str)
@pytest.mark.parametrize("gt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("beta", [0.999, 0.9999, 0.999999])
def test_orthogonal_step_with_beta_near_one(dev, heads, shape, gt, beta):
    """1 - beta is that of the caller's beta, not of its rounding: momentum within four roundings."""
    gen = torch.Generator().manual_seed(1)
    grad, w = torch.randn(shape, generator=gen).to(gt), torch.randn(shape, generator=gen)
    for mom in (torch.zeros(shape), 1e-4 * torch.randn(shape, generator=gen)):
        for nesterov in (True, False):
            _, om = heads.orthogonal_step(w.to(dev), grad.to(dev), mom.to(dev), 0.1, beta, nesterov)
            new = beta * mom.double() + (1 - beta) * grad.double()
            within(om, new, 4 * UNIT[F32] * (beta * mom.double().abs() + (1 - beta) * grad.double().abs()))
            if shape == (90, 128):
                ow, _ = heads.orthogonal_step(w.to(dev), grad.to(dev), mom.to(dev), 0.1, beta, nesterov)
                d = beta * new + (1 - beta) * grad.double() if nesterov else new
                o = ortho_exact(d, 5, QUINTIC, 1e-7)
                noise = max(float(torch.linalg.vector_norm(ortho_exact(d, 5, QUINTIC, 1e-7, 2.0 ** -21, k) - o)) for k in range(3))
                want = w.double() - 0.1 * o
                assert float(torch.linalg.vector_norm(f64(ow) - want)) <= 0.8 * noise + 2 * UNIT[F32] * float(
                    torch.linalg.vector_norm(want)) + 1e-7


# ---------------------------------------------------------------- norms below eps
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,m,n", [(1, 40, 50), (1, 100, 130), (2, 300, 210), (5, 1030, 1100)])
def test_orthogonalize_far_below_eps(dev, heads, dtype, batch, m, n):
    """Norms of eps times 1 to 1e-20: the iteration keeps its precision while it
    lifts them."""
    gen = torch.Generator().manual_seed(m)
    base = torch.randn(m, n, generator=gen)
    base /= torch.linalg.vector_norm(base)
    few = batch == 5
    for eps in ((1e-7,) if few else (1e-7, 1.0)):
        for ratios, steps, coef in (((1.0, 1e-2, 1e-4, 1e-7, 1e-10), 5, QUINTIC), ((0.3, 1e-3, 1e-5, 1e-12, 1e-20), 14, QUINTIC),
                                    ((0.1, 1e-4, 1e-6, 1e-8, 1e-9), 4, [(0.5, 0.1, 0.1), POLAR, (8.0, -3.0, 1.0), (64.0, 1.0, -1.0)])):
            if few and steps != 5:
                continue
            for k in range(0, len(ratios), batch):
                r = ratios[k:k + batch]
                g = torch.stack([base * (eps * v) for v in r]).to(dtype)
                got = heads.orthogonalize(g.to(dev), steps=steps, coefficients=coef, eps=eps)
                for i in range(len(r)):
                    if few and i not in (0, 3):
                        continue
                    check_ortho(heads, got[i], g[i].double(), dtype, steps, coef, eps)


# ---------------------------------------------------------------- norms at the ends of the range
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(12, 40), (64, 9), (150, 90), (100, 128)])
def test_orthogonalize_norms_at_the_ends_of_the_range(dev, heads, dtype, m, n):
    """Matrices of the smallest and the largest finite numbers."""
    gen = torch.Generator().manual_seed(n)
    base = torch.randn(m, n, generator=gen)
    for size, eps in ((1e-36, 1e-30), (1e-38, 1e-30), (1e-40, 1e-30), (2.0 ** -126, 1e-7), (1e36, 1e-7), (6e37, 1e-7), (6e37, 1.0)):
        g = (base * size).to(dtype)
        assert torch.isfinite(g).all()
        got = heads.orthogonalize(g.to(dev), eps=eps)
        check_ortho(heads, got, g.double(), dtype, 5, QUINTIC, eps)


# ---------------------------------------------------------------- rows at the ends of the range
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("g", [3, 80])
@pytest.mark.parametrize("px,pw", [(118, -30), (100, 0), (0, 100), (0, 80), (-110, 30), (-100, 20), (-60, 100), (60, -40)])
def test_adapted_rows_at_the_ends_of_the_range(dev, heads, dtype, n, g, px, pw):
    """Rows of x, dy and W whose sizes are far from one, their products inside FP32's range."""
    t, a, s, bias = adapted_case(dev, dtype, n, 72, 40, g, 4, "mixed", seed=11)
    x, W = t["x"].clone(), t["W"].clone()
    t["x"][::2] = (x[::2].float() * 2.0 ** px).to(dtype)
    t["W"] = (W.float() * 2.0 ** pw).to(dtype)
    t["B"] = (t["B"].float() * 2.0 ** min(pw, 0)).to(dtype)
    y, ty = (v[0] for v in adapted_exact(t, a, s, None))
    within(heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, scales=s), y, tolerance(dtype, y, ty, 76), "y")
    t["x"] = x
    t["dy"][::2] = (t["dy"][::2].float() * 2.0 ** px).to(dtype)
    t["A"] = (t["A"].float() * 2.0 ** min(pw, 0)).to(dtype)
    dx, tdx = (v[1] for v in adapted_exact(t, a, s, None))
    got = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s, need_dA=False, need_dB=False)
    within(got[0], dx, tolerance(dtype, dx, tdx, 44), "dx")


# ---------------------------------------------------------------- huge factors
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 300])
@pytest.mark.parametrize("size,pw", [(3.39e38, 0), (2.0 ** 75, -70), (2.0 ** 66, -40)])
def test_adapted_large_factors_stay_apart(dev, heads, dtype, n, size, pw):
    """Huge finite values in one adapter reach the outputs of its rows, and no other."""
    t, a, s, _ = adapted_case(dev, dtype, n, 136, 88, 3, 8, "mixed", seed=9)
    a[:3] = torch.tensor([0, 1, -1], dtype=torch.int32)
    t["W"][5] = (t["W"][5].float() * 2.0 ** pw).to(dtype)
    clean = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, scales=s)
    back = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)
    A, B = t["A"].clone(), t["B"].clone()
    B[0, 5] = size
    A[0, :, 7] = size
    other = (a != 0).to(dev)
    got = heads.adapted_logits(t["x"], t["W"], t["A"], B, a, scales=s)
    assert torch.equal(got[other], clean[other])
    keep = torch.arange(88, device=dev) != 5
    assert torch.equal(got[:, keep], clean[:, keep])
    dx, dA, dB = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], A, t["B"], a, scales=s)
    assert torch.equal(dx[other], back[0][other]) and torch.equal(dA, back[1]) and torch.equal(dB[1:], back[2][1:])
    keep = torch.arange(136, device=dev) != 7
    assert torch.equal(dx[:, keep], back[0][:, keep])
    # and there, where FP32 holds it, the product itself
    t2 = dict(t, B=B)
    y, ty = (v[0] for v in adapted_exact(t2, a, s, None))
    y, ty, got = y[:, 5], ty[:, 5], f64(got[:, 5])
    fits = ty < 2.0 ** 127
    within(got[fits], y[fits], tolerance(dtype, y, ty, 144)[fits], "y")


# ---------------------------------------------------------------- a head that is not finite
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 300])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_adapted_non_finite_head_stays_in_its_places(dev, heads, dtype, n, bad):
    """An infinity or a NaN in W reaches its class's logits and its feature's gradient, and no other."""
    t, a, s, _ = adapted_case(dev, dtype, n, 72, 40, 3, 4, "mixed", seed=13)
    t["W"] = (t["W"].float() * 2.0 ** -30).to(dtype)
    t["A"] = (t["A"].float() * 2.0 ** -30).to(dtype)
    want = [v[:2] for v in adapted_exact(t, a, s, None)]
    W = t["W"].clone()
    W[3, 9] = bad
    y = heads.adapted_logits(t["x"], W, t["A"], t["B"], a, scales=s)
    dx = heads.adapted_logits_backward(t["dy"], t["x"], W, t["A"], t["B"], a, scales=s, need_dA=False, need_dB=False)[0]
    for got, k, K, at in ((y, 0, 76, 3), (dx, 1, 44, 9)):
        assert not torch.isfinite(got[:, at]).any()
        w, terms = want[0][k], want[1][k]
        keep = torch.arange(w.shape[1]) != at
        within(got[:, keep.to(dev)], w[:, keep], tolerance(dtype, w, terms, K)[:, keep], str(k))


# ---------------------------------------------------------------- autograd
def test_tensors_that_require_gradients(dev, heads):
    x, W = torch.randn(4, 16, device=dev), torch.randn(8, 16, device=dev)
    A, B = torch.randn(2, 3, 16, device=dev), torch.randn(2, 8, 3, device=dev)
    ids = torch.zeros(4, dtype=torch.int32, device=dev)
    bias, scales, dy = torch.randn(8, device=dev), torch.rand(2, device=dev), torch.randn(4, 8, device=dev)
    named = dict(x=x, W=W, A=A, B=B, bias=bias, scales=scales)
    heads.adapted_logits(adapter=ids, **named)
    for name, t in named.items():
        leaf = dict(named, **{name: t.clone().requires_grad_()})
        with pytest.raises(ValueError, match=name):
            heads.adapted_logits(adapter=ids, **leaf)
        with torch.no_grad():
            heads.adapted_logits(adapter=ids, **leaf)
        if name != "bias":
            leaf.pop("bias")
            with pytest.raises(ValueError, match=name):
                heads.adapted_logits_backward(dy, adapter=ids, **leaf)
    with pytest.raises(ValueError, match="out"):
        heads.adapted_logits(adapter=ids, out=torch.empty(4, 8, device=dev).requires_grad_(), **named)
    with pytest.raises(ValueError, match="dy"):
        heads.adapted_logits_backward(dy.clone().requires_grad_(), x, W, A, B, ids)
    with pytest.raises(ValueError, match="logits"):
        heads.cross_entropy(x.clone().requires_grad_(), ids)
    with pytest.raises(ValueError, match="weight"):
        heads.cross_entropy(x, ids, torch.ones(4, device=dev).requires_grad_())
    with pytest.raises(ValueError, match="G"):
        heads.orthogonalize(x.clone().requires_grad_())
    for k in range(3):
        args = [x.clone(), x.clone(), x.clone()]
        args[k].requires_grad_()
        with pytest.raises(ValueError):
            heads.orthogonal_step(*args, 0.1)
        with torch.no_grad():
            heads.orthogonal_step(*args, 0.1)


# ---------------------------------------------------------------- writes in place
def test_writes_in_place_are_seen(dev, heads):
    """What a call overwrites counts as changed, so that a gradient that needs the old values says so."""
    x, W = torch.randn(4, 16, device=dev), torch.randn(8, 16, device=dev)
    A, B = torch.randn(2, 3, 16, device=dev), torch.randn(2, 8, 3, device=dev)
    ids, out = torch.zeros(4, dtype=torch.int32, device=dev), torch.empty(4, 8, device=dev)
    heads.adapted_logits(x, W, A, B, ids, out=out)
    assert out._version == 1
    heads.cross_entropy(out, ids, in_place=True)
    assert out._version == 2
    heads.cross_entropy(out, ids)
    assert out._version == 2
    o = torch.empty_like(x)
    heads.orthogonalize(x, out=o)
    assert o._version == 1 and x._version == 0
    w, m, g = x.clone(), x.clone(), x.clone()
    was = [t._version for t in (w, m, g)]
    heads.orthogonal_step(w, g, m, 0.1)
    assert [t._version for t in (w, m, g)] == [was[0] + 1, was[1] + 1, was[2]]
    heads.orthogonal_step(w, g, m, 0.1, out=(o, torch.empty_like(x)))
    assert o._version == 2 and w._version == was[0] + 1
    leaf = torch.nn.Parameter(x.clone())
    y = (leaf * leaf).sum()
    with torch.no_grad():
        heads.orthogonal_step(leaf, g, m, 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():
        heads.orthogonal_step(w.clone(), g, m.clone(), 0.1)
        heads.adapted_logits(x, W, A, B, ids, out=torch.empty(4, 8, device=dev))


# ---------------------------------------------------------------- messages of refusals
def test_refusals_say_why_every_time(dev, heads):
    from paper_2608_13144_gb300 import LipCacheError
    x, W = torch.randn(4, 16, device=dev), torch.randn(8, 16, device=dev)
    ids = torch.zeros(4, dtype=torch.int32, device=dev)
    for _ in range(2):
        with pytest.raises(LipCacheError, match="rank"):
            heads.adapted_logits(x, W, x.new_zeros(2, 129, 16), x.new_zeros(2, 8, 129), ids)
        with pytest.raises(LipCacheError, match="rank"):
            heads.adapted_logits_backward(x.new_zeros(4, 8), x, W, x.new_zeros(2, 129, 16), x.new_zeros(2, 8, 129), ids)
        with pytest.raises(LipCacheError, match="rows and cols"):
            heads.orthogonalize(x.new_zeros(0, 8))


# ---------------------------------------------------------------- coefficients
def test_coefficients_of_any_sequences(dev, heads):
    g = torch.randn(20, 30, device=dev)
    want = heads.orthogonalize(g, steps=2, coefficients=[QUINTIC, POLAR])
    for co in ((QUINTIC, POLAR), ([*QUINTIC], [*POLAR]), [[*QUINTIC], [*POLAR]], (*QUINTIC, *POLAR),
               torch.tensor([QUINTIC, POLAR], dtype=torch.float64)):
        assert torch.equal(heads.orthogonalize(g, steps=2, coefficients=co), want)
    one = heads.orthogonalize(g, steps=2, coefficients=QUINTIC)
    for co in ([*QUINTIC], ([*QUINTIC],), (QUINTIC,), [QUINTIC] * 2, tuple(torch.tensor(QUINTIC, dtype=torch.float64))):
        assert torch.equal(heads.orthogonalize(g, steps=2, coefficients=co), one)
    # numbers in tensors that change between calls
    co = tuple(torch.tensor(v, dtype=torch.float64) for v in QUINTIC)
    assert torch.equal(heads.orthogonalize(g, steps=2, coefficients=co), one)
    for c, v in zip(co, POLAR):
        c.fill_(v)
    assert torch.equal(heads.orthogonalize(g, steps=2, coefficients=co), heads.orthogonalize(g, steps=2, coefficients=POLAR))


# ---------------------------------------------------------------- sizes past 32 bits
def test_sizes_past_32_bits_are_refused(dev, heads):
    """Not cut off to their lowest 32 bits (8 classes, 8 columns here)."""
    one = torch.zeros(1, 1, dtype=BF16, device=dev)
    wide = one.expand(1, 2 ** 32 + 8)
    ids = torch.zeros(1, dtype=torch.int32, device=dev)
    none = one.new_empty(0, 1, 1)
    for call in (lambda: heads.cross_entropy(wide, ids), lambda: heads.orthogonalize(wide),
                 lambda: heads.orthogonal_step(wide, wide, wide, 0.1),
                 lambda: heads.adapted_logits(wide, wide, none.expand(0, 1, 2 ** 32 + 8), none, ids)):
        with pytest.raises(ValueError, match="2147483647"):
            call()
