"""log_probs, log_probs_backward and distill, through the binding, against plain
64-bit forms on the CPU.

Tolerances, u = 2^-24. With x = (max - z) / T, a term exp(-x) of a row's sum is
off by 3 u x (difference, factor, product) and 2^-22 (the special function unit)
of itself; a thread adds at most L = C / 512 + 128 of them in two chains,
rescaled by 2^-22 at most every 16, and 12 additions join the threads'. All terms
are positive, so that the sum is within B = u (L + 64 + 4 mean x) of itself, and its
logarithm within B, or 20 B of itself where it is below 1 / 20. The mean of x is off
by that and by 3 u x in each term's x. Each result adds a few roundings of its own.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
BOTH = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
U = 2.0 ** -24
INF = math.inf


def half(dtype):
    return torch.finfo(dtype).eps / 2


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
    return heads


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


class Exact:
    """Of rows of logits: m, x, p, log_sum, mean, entropy and lp in 64 bits, with their tolerances."""

    def __init__(self, z, T):
        z = f64(z)
        n, c = z.shape
        self.z, self.T = z, T
        self.bad = torch.isnan(z).any(1) | (z == INF).any(1)
        self.m = z.amax(1)
        self.none = ~self.bad & (self.m == -INF)
        self.live = ~(self.bad | self.none)
        m = torch.where(self.live, self.m, torch.zeros_like(self.m))
        zz = torch.where(self.live[:, None], z, torch.zeros_like(z))
        self.x = (m[:, None] - zz) / T
        e = torch.exp(-self.x)
        others = e.clone()
        others[torch.arange(n), zz.argmax(1)] = 0.0
        others = others.sum(1)
        self.log_sum = torch.log1p(others)
        self.p = e / (1 + others)[:, None]
        px = torch.where(e > 0, self.p * self.x, torch.zeros_like(e))
        self.mean = px.sum(1)
        second = torch.where(e > 0, px * self.x, torch.zeros_like(e)).sum(1)
        B = U * (c / 512 + 128 + 64 + 4 * self.mean)
        # (terms below 2^-126, of x from 87 on, are flushed to 0 by the special function unit: c of them at
        # most, and x exp(-x) falls from there)
        flushed = c * 2.0 ** -126
        self.tol_sum = B * torch.clamp(20 * self.log_sum, max=1.0) + 4 * U * self.log_sum + flushed
        self.tol_mean = 3 * U * second + (B + 8 * U) * self.mean + 88 * flushed
        self.lp = -self.x - self.log_sum[:, None]
        self.tol_lp = 3 * U * self.x + 2 * U * self.lp.abs() + self.tol_sum[:, None]
        fill = torch.where(self.bad, math.nan, -INF).double()
        self.lp[~self.live] = fill[~self.live][:, None]
        self.entropy = self.log_sum + self.mean
        for t in (self.log_sum, self.mean, self.entropy, self.m):
            t[self.bad] = math.nan
        for t in (self.log_sum, self.mean, self.entropy):
            t[self.none] = 0.0


def target_lp(ex, y):
    """(logprob, its tolerance) of the targets y."""
    n, c = ex.z.shape
    ok = (y >= 0) & (y < c)
    at = torch.where(ok, y, torch.zeros_like(y))[:, None]
    lp, tol = ex.lp.gather(1, at)[:, 0], ex.tol_lp.gather(1, at)[:, 0]
    return torch.where(ok, lp, torch.zeros_like(lp)), tol


def check_answers(heads, z, y, k, T=1.0):
    ex = Exact(z, T)
    before = z.clone()
    r = heads.log_probs(z, y, top=k, temperature=T)
    lp, tol = target_lp(ex, y.cpu().long())
    within(r.logprob, lp, tol, "logprob")
    within(r.entropy, ex.entropy, ex.tol_sum + ex.tol_mean + U * ex.entropy.abs(), "entropy")
    within(r.norm[:, 0], ex.m, torch.zeros(1, dtype=torch.float64), "max")
    within(r.norm[:, 1], ex.log_sum, ex.tol_sum, "log_sum")
    within(r.norm[:, 2], ex.mean, ex.tol_mean, "mean")
    assert torch.equal(torch.nan_to_num(z), torch.nan_to_num(before))
    if not k:
        assert r.top is None and r.index is None
        return r
    n, c = z.shape
    w = min(k, c)
    order = torch.sort(ex.z + 0.0, dim=1, descending=True, stable=True).indices[:, :w]
    there = (ex.z.gather(1, order) > -INF) & ex.live[:, None]
    index = torch.full((n, k), -1)
    index[:, :w] = torch.where(there, order, torch.full_like(order, -1))
    assert torch.equal(r.index.cpu().long(), index), "index"
    top, tol = torch.full((n, k), -INF, dtype=torch.float64), torch.zeros(n, k, dtype=torch.float64)
    top[:, :w] = torch.where(there, ex.lp.gather(1, order), torch.full_like(order, -INF, dtype=torch.float64))
    tol[:, :w] = ex.tol_lp.gather(1, order)
    top[ex.bad] = math.nan
    within(r.top, top, tol, "top")
    return r


def logits(dev, dtype, n, c, seed=0, spread=3.0):
    gen = torch.Generator().manual_seed(seed + 31 * n + c)
    z = spread * torch.randn(n, c, generator=gen)
    y = torch.randint(0, c, (n,), generator=gen)
    y[torch.rand(n, generator=gen) < 0.1] = -1
    return z.to(dtype).to(dev), y.int().to(dev)


SIZES = [(1, 1, 1), (1, 2, 2), (3, 10, 5), (2, 33, 40), (7, 200, 5), (5, 255, 32), (4, 257, 33), (9, 1000, 20),
         (6, 1023, 128), (3, 2047, 8), (5, 2049, 64), (2, 4096, 1), (3, 8200, 128), (2, 16_390, 20), (2, 20_001, 50),
         (3, 50_001, 20), (1, 131_073, 100), (1, 400_003, 7), (700, 200, 10), (300, 17, 3), (64, 3000, 0), (40, 12_345, 16),
         (30, 140_000, 128), (41, 140_001, 30), (200, 7000, 32), (160, 7001, 33), (33, 31_000, 65)]


@BOTH
@pytest.mark.parametrize("n,c,k", SIZES, ids=lambda v: str(v))
def test_answers(dev, heads, dtype, n, c, k):
    z, y = logits(dev, dtype, n, c)
    check_answers(heads, z, y, k, T={0: 1.0, 1: 0.5, 2: 4.0}[(n + c) % 3])


@BOTH
@pytest.mark.parametrize("c", [40, 200, 1500, 9000, 60_000])
def test_answers_where_values_repeat(dev, heads, dtype, c):
    """Rows all equal, of few values, in rising and falling order, with the large ones side by side or far apart."""
    gen = torch.Generator().manual_seed(c)
    rows = [torch.zeros(c), torch.full((c,), -2.5), torch.randint(0, 3, (c,), generator=gen).float(),
            torch.randint(-1, 1, (c,), generator=gen).float() * 0.0,  # 0 and -0
            torch.arange(c).float(), -torch.arange(c).float(),
            torch.where(torch.arange(c) < c // 2, 1.0, 1.0 + 2 ** -7),
            torch.where(torch.arange(c) % 97 == 5, 4.0, torch.randn(c, generator=gen)),
            torch.where((torch.arange(c) - c // 3).abs() < 900, 5.0 + torch.rand(c, generator=gen), 0.0)]
    z = torch.stack(rows).to(dtype).to(dev)
    y = torch.arange(len(rows), device=dev).int()
    for k in (1, 13, 32, 128):
        check_answers(heads, z, y, k)


@BOTH
@pytest.mark.parametrize("c", [64, 200, 3001, 30_000])
def test_answers_of_masked_and_odd_rows(dev, heads, dtype, c):
    low = torch.finfo(dtype).min
    z, _ = logits(dev, dtype, 14, c, seed=3)
    y = torch.full((14,), c // 2, dtype=torch.int32, device=dev)
    z[0] = -INF
    z[1] = -INF
    z[1, c // 2] = -7.0  # one class left
    z[2, ::2] = -INF
    z[3] = low
    z[4, 1:] = low
    z[5, 3] = math.nan
    z[6, c - 1] = INF
    z[7, c - 1] = -math.nan
    z[8, :] = math.nan
    z[9, 5:] = -INF
    z[9, c // 2] = -INF  # a masked target
    z[10, :], z[10, c - 1], z[10, 0] = -INF, low, low
    z[11] = torch.finfo(dtype).max
    z[12, c // 2] = torch.finfo(dtype).max
    y[13] = c  # outside
    y[5] = -1  # ignored, and NaN
    check_answers(heads, z, y, 9, T=2.0)
    check_answers(heads, z, y, 40)


@BOTH
@pytest.mark.parametrize("c", [10, 200, 9000])
def test_sure_rows_keep_their_precision(dev, heads, dtype, c):
    """The logarithm of a sure class is that of the others' share, wherever the logits stand."""
    z, y = logits(dev, dtype, 6, c, seed=8, spread=1.0)
    z = z.float()
    for i, gap in enumerate((4.0, 8.0, 16.0, 24.0, 40.0, 80.0)):
        y[i] = (i * 7) % c
        z[i, y[i]] = z[i].max() + gap + math.log(c)
    check_answers(heads, z.to(dtype), y, 4)
    check_answers(heads, (z + 1000.0).to(dtype), y, 4, T=0.5)
    r = heads.log_probs(z.to(dtype), y)
    assert (r.logprob[:4] < 0).all()  # not rounded to 0
    dz = heads.log_probs_backward(z.to(dtype), r.norm, y, torch.ones(6, device=dev))
    own = f64(dz).gather(1, y.cpu().long()[:, None])[:, 0]
    ex = Exact(z.to(dtype), 1.0)
    want = -torch.expm1(ex.lp.gather(1, y.cpu().long()[:, None])[:, 0])
    within(own, want, want * (half(dtype) + 2 ** -16) + c * 2.0 ** -126)


@BOTH
@pytest.mark.parametrize("n,c", [(3, 57), (2, 203), (3, 2500), (2, 17_001)])
def test_strides_and_offsets(dev, heads, dtype, n, c):
    """Rows of wider matrices, off the 16-byte boundaries, with NaN beside them."""
    z0, y = logits(dev, dtype, n, c, seed=5)
    g, h = torch.randn(n, device=dev), torch.randn(n, device=dev)
    for left, right in ((0, 1), (1, 0), (3, 2), (8, 8), (5, 11)):
        w = torch.full((n, left + c + right), math.nan, dtype=dtype, device=dev)
        z = w[:, left:left + c]
        z.copy_(z0)
        r = check_answers(heads, z, y, 12)
        top, index = torch.randn(n, 4, device=dev), torch.tensor([[0, c - 1, c // 2, c]] * n, dtype=torch.int32, device=dev)
        check_gradient(heads, z, y, g, h)
        check_distill(heads, z, top, index, None)
        for call in (lambda: heads.log_probs_backward(z, r.norm, y, g, h, in_place=True),
                     lambda: heads.distill(z, top, index, in_place=True)[1]):
            z.copy_(z0)
            keep = w.clone()
            version = z._version
            assert call().data_ptr() == z.data_ptr() and z._version > version
            assert torch.isnan(w[:, :left]).all() and torch.isnan(w[:, left + c:]).all()
            assert not torch.equal(keep[:, left:left + c], z)
    z, wide = z0.repeat_interleave(2, 1)[:, ::2], z0.t().contiguous().t()  # copied first
    for v in (z, wide):
        assert torch.equal(heads.log_probs(v, y).norm, heads.log_probs(z0, y).norm)


# ---------------------------------------------------------------- gradient of the log-probabilities
def check_gradient(heads, z, y, g, h, T=1.0):
    ex = Exact(z, T)
    norm = heads.log_probs(z, y, temperature=T).norm
    dz = heads.log_probs_backward(z, norm, y, g, h, temperature=T)
    assert dz.dtype == z.dtype
    n, c = z.shape
    zero = torch.zeros(n, dtype=torch.float64)
    y = torch.full((n,), -1) if y is None else y.cpu().long()
    ok = (y >= 0) & (y < c)
    g, h = (zero if g is None else torch.where(ok, f64(g), zero))[:, None], (zero if h is None else f64(h))[:, None]
    hot = torch.zeros(n, c, dtype=torch.float64)
    hot[torch.arange(n)[ok], y[ok]] = 1.0
    p = torch.where(ex.live[:, None], ex.p, torch.zeros_like(ex.p))
    x = torch.where(p > 0, ex.x, torch.zeros_like(ex.x))
    mean = torch.where(ex.live, ex.mean, zero)[:, None]
    want = (g * (hot - p) - h * p * (mean - x)) / T
    # p by its exponent, the factor by log_sum's, the special function unit twice
    rel = U * (3 * x + 4 * torch.nan_to_num(ex.log_sum)[:, None] + 24) + torch.nan_to_num(ex.tol_sum)[:, None]
    tol = (p * (g.abs() + h.abs() * (x + mean)) * (rel + 8 * U) + h.abs() * p * torch.nan_to_num(ex.tol_mean)[:, None]
           + g.abs() * hot * (1 - p) * 8 * U) / T
    want[ex.none] = 0.0
    want[ex.bad] = math.nan
    want[((g == 0) & (h == 0))[:, 0]] = 0.0
    within(dz, want, tol + half(z.dtype) * want.abs() + 1e-36, "dz")
    return dz


@BOTH
@pytest.mark.parametrize("n,c", [(1, 1), (3, 2), (5, 33), (9, 200), (130, 513), (4, 4099), (2, 50_001), (1500, 10)])
def test_gradient(dev, heads, dtype, n, c):
    z, y = logits(dev, dtype, n, c, seed=2)
    gen = torch.Generator().manual_seed(n)
    g, h = torch.randn(n, generator=gen).to(dev), torch.randn(n, generator=gen).to(dev)
    for T in (1.0, 0.7, 3.0):
        check_gradient(heads, z, y, g, h, T)
    check_gradient(heads, z, y, g, None)
    check_gradient(heads, z, None, None, h)
    check_gradient(heads, z, None, None, None)


@BOTH
def test_gradient_of_masked_and_odd_rows(dev, heads, dtype):
    c = 300
    z, y = logits(dev, dtype, 8, c, seed=4)
    y[:] = 7
    z[0], z[1, 2:], z[2, 9], z[3, 9] = -INF, -INF, math.nan, INF
    z[4] = torch.finfo(dtype).min
    z[5, 8:] = torch.finfo(dtype).min
    y[6] = -1
    z[6, 0] = math.nan
    g, h = torch.ones(8, device=dev), torch.ones(8, device=dev)
    check_gradient(heads, z, y, g, h)
    check_gradient(heads, z, y, g, None)  # row 6: nothing asked for, whatever its logits
    check_gradient(heads, z, y, g * 0, h * 0)


@BOTH
def test_gradients_against_differences(dev, heads, dtype):
    """sum(g logprob + h entropy) and the sum of distill's losses along a direction, by 64-bit differences of the
    formulas, against the gradients' products with it."""
    n, c, T = 6, 150, 1.7
    z, y = logits(dev, dtype, n, c, seed=12, spread=1.5)
    gen = torch.Generator().manual_seed(5)
    g, h, step = (torch.randn(*s, generator=gen).double() for s in ((n,), (n,), (n, c)))
    top, index = torch.randn(n, 6, generator=gen), torch.randint(0, c, (n, 6), generator=gen)
    w = torch.rand(n, generator=gen).double()
    q = torch.softmax(top.double() / T, 1)

    def policy(v):
        lp = torch.log_softmax(v / T, 1)
        ok = (y.cpu() >= 0).double()
        given = lp.gather(1, y.cpu().long().clamp(min=0)[:, None])[:, 0]
        return float((g * ok * given - h * (lp.exp() * lp).sum(1)).sum())

    def student(v):
        lp = torch.log_softmax(v / T, 1)
        # (classes named twice: their shares add up)
        dense = torch.zeros(n, c, dtype=torch.float64).scatter_add_(1, index, q)
        return float((w * T * T * (torch.xlogy(dense, dense) - dense * lp).sum(1)).sum())

    r = heads.log_probs(z, y, temperature=T)
    grads = {policy: heads.log_probs_backward(z, r.norm, y, g.float().to(dev), h.float().to(dev), temperature=T),
             student: heads.distill(z, top.to(dev), index.int().to(dev), w.float().to(dev), temperature=T)[1]}
    e = 1e-5
    for f, d in grads.items():
        diff = (f(f64(z) + e * step) - f(f64(z) - e * step)) / (2 * e)
        # outputs' rounding, 2^-18 of their own, and the differences' 1e-6
        size = float((f64(d).abs() * step.abs()).sum())
        assert abs(diff - float((f64(d) * step).sum())) <= (half(dtype) + 2 ** -18) * size + 1e-6


# ---------------------------------------------------------------- distillation
def check_distill(heads, z, top, index, w, T=1.0, **kw):
    ex = Exact(z, T)
    n, c = z.shape
    k = top.shape[1]
    loss, dz = heads.distill(z, top, index, w, temperature=T, **kw)
    v, idx = f64(top), index.cpu().long()
    w = torch.ones(n, dtype=torch.float64) if w is None else f64(w)
    ok = (idx >= 0) & (idx < c)
    v = torch.where(ok, v, torch.full_like(v, -INF))
    odd = torch.isnan(v).any(1) | (v == INF).any(1)
    none = (v == -INF).all(1) | (w == 0)
    v[odd | none] = 0.0
    xq = (v.amax(1, keepdim=True) - v) / T
    q = torch.softmax(-xq, 1)
    lq = torch.log_softmax(-xq, 1)
    at = torch.where(ok, idx, torch.zeros_like(idx))
    lp, tol_lp = ex.lp.gather(1, at), ex.tol_lp.gather(1, at)
    has = q > 0
    zero = torch.zeros_like(q)
    gap = torch.where(has, lq - lp, zero)
    rq = U * (4 * xq + k + 24)
    want = w * T * T * torch.where(has, q * gap, zero).sum(1)
    part = q * (rq * (gap.abs() + 1) + 6 * U * (lq.abs() + lp.abs()) + tol_lp + 12 * U * gap.abs())
    tol = w.abs() * T * T * torch.where(has, part, zero).sum(1) + 4 * U * want.abs()
    p = torch.where(ex.live[:, None], ex.p, torch.zeros_like(ex.p))
    share = torch.zeros(n, c, dtype=torch.float64).scatter_add_(1, at, torch.where(ok, q, zero))
    err = torch.zeros(n, c, dtype=torch.float64).scatter_add_(1, at, torch.where(ok & has, q * rq, zero))
    x = torch.where(p > 0, ex.x, torch.zeros_like(p))
    rel = U * (3 * x + 24) + torch.nan_to_num(ex.tol_sum)[:, None] + U * (c / 512 + 200) + 4 * U * torch.nan_to_num(ex.log_sum)[:, None]
    grad = (w * T)[:, None] * (p - share)
    bound = (w * T).abs()[:, None] * (p * rel + err) + half(z.dtype) * grad.abs() + 1e-36
    want[ex.none] = INF
    want[ex.bad | odd] = grad[ex.bad | odd] = math.nan
    want[none] = grad[none] = 0.0
    grad[ex.none] = 0.0
    tol[none], bound[none] = 0.0, 0.0
    within(loss, want, tol + 1e-36, "loss")
    if dz is not None:
        assert dz.dtype == z.dtype
        within(dz, grad, bound, "dz")
    return loss, dz


def teacher(dev, z, k, seed=0):
    """A teacher's k classes of each row: near the student's own best."""
    gen = torch.Generator().manual_seed(seed + k)
    n, c = z.shape
    best = (0.7 * z.float().cpu() + torch.randn(n, c, generator=gen)).topk(min(k, c), 1)
    top, index = torch.full((n, k), 3.0), torch.full((n, k), -1)
    top[:, :min(k, c)], index[:, :min(k, c)] = best.values, best.indices
    index[torch.rand(n, k, generator=gen) < 0.1] = -1
    return top.to(dev), index.int().to(dev)


@BOTH
@pytest.mark.parametrize("n,c,k", [s for s in SIZES if s[2]], ids=lambda v: str(v))
def test_distill(dev, heads, dtype, n, c, k):
    z, _ = logits(dev, dtype, n, c, seed=6)
    top, index = teacher(dev, z, k)
    w = torch.rand(n, generator=torch.Generator().manual_seed(n)).to(dev)
    check_distill(heads, z, top, index, w, T={0: 1.0, 1: 0.5, 2: 4.0}[(n + c) % 3])
    check_distill(heads, z, top, index, None, need_grad=False)


@BOTH
def test_distill_same_class_twice(dev, heads, dtype):
    for c, k in ((5, 12), (300, 40), (5000, 100)):
        z, _ = logits(dev, dtype, 9, c, seed=7)
        gen = torch.Generator().manual_seed(k)
        top = torch.randn(9, k, generator=gen).to(dev)
        index = torch.randint(-1, min(c, 7) + 1, (9, k), generator=gen).int().to(dev)
        check_distill(heads, z, top, index, None, T=1.5)


@BOTH
@pytest.mark.parametrize("c", [100, 1000, 9000])
def test_distill_of_masked_and_odd_rows(dev, heads, dtype, c):
    z, _ = logits(dev, dtype, 16, c, seed=9)
    top = torch.randn(16, 5, generator=torch.Generator().manual_seed(1)).to(dev)
    index = torch.tensor([[1, 4, c - 1, 9, 2]] * 16, dtype=torch.int32, device=dev)
    w = torch.full((16,), 0.5, device=dev)
    z[0] = -INF
    z[1, 4] = -INF  # a masked class with a share: loss +inf
    z[2, 4], top[2, 1] = -INF, -INF  # without one
    z[3, 8], z[4, 8] = math.nan, INF
    index[5] = -1  # no teacher
    z[5, 3] = math.nan
    index[6, :4] = c  # one class left
    w[7] = 0.0
    z[7, 3] = math.nan
    top[8] = -INF
    top[9, 2], top[10, 2] = math.nan, INF
    top[11, 2], index[11, 2] = math.nan, -1  # left out
    z[12] = torch.finfo(dtype).min
    z[13, 10:] = -INF
    z[13, 2] = -INF
    index[13, 2], index[13, 4] = 3, 5
    top[14] = -1e30
    top[15, 0], top[15, 1] = 1e30, -1e30
    check_distill(heads, z, top, index, w)


@BOTH
def test_distill_of_sure_rows(dev, heads, dtype):
    """Where student and teacher are sure of one class, its gradient is the difference of what they leave to others."""
    c = 64
    z, _ = logits(dev, dtype, 5, c, seed=10, spread=1.0)
    z = z.float()
    z[torch.arange(5), torch.arange(5)] = z.amax(1) + torch.tensor([8.0, 10.0, 12.0, 14.0, 16.0], device=dev)
    z = z.to(dtype)
    top = torch.tensor([[30.0, 0.0, 20.0]] * 5, device=dev)
    index = torch.tensor([[i, i + 9, i + 20] for i in range(5)], dtype=torch.int32, device=dev)
    _, dz = check_distill(heads, z, top, index, None)
    ex = Exact(z, 1.0)
    left = math.exp(-30.0) + math.exp(-10.0)
    at = torch.arange(5)
    own = -(-torch.expm1(ex.lp[at, at])) + left / (1 + left)  # p - q = (1 - q) - (1 - p)
    within(f64(dz)[at, at], own, own.abs() * half(dtype) + 2 ** -16 * (-torch.expm1(ex.lp[at, at]) + left))


# ---------------------------------------------------------------- calls
@BOTH
def test_empty_batches(dev, heads, dtype):
    z, y = torch.empty(0, 30, dtype=dtype, device=dev), torch.empty(0, dtype=torch.int32, device=dev)
    r = heads.log_probs(z, y, top=3)
    assert r.logprob.shape == r.entropy.shape == (0,) and r.norm.shape == (0, 3) and r.top.shape == r.index.shape == (0, 3)
    assert heads.log_probs_backward(z, r.norm, y, r.logprob).shape == (0, 30)
    loss, dz = heads.distill(z, r.top, r.index)
    assert loss.shape == (0,) and dz.shape == (0, 30)


@BOTH
@pytest.mark.parametrize("n,c", [(500, 200), (60, 5000), (3, 60_000)])
def test_repeats_on_streams_and_in_graphs(dev, heads, dtype, n, c):
    z, y = logits(dev, dtype, n, c, seed=11)
    top, index = teacher(dev, z, 16)
    g = torch.randn(n, device=dev)

    def all_of(z):
        r = heads.log_probs(z, y, top=16, temperature=0.8)
        return (*r, heads.log_probs_backward(z, r.norm, y, g, g, temperature=0.8), *heads.distill(z, top, index, temperature=2.0))

    want = all_of(z)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, all_of(z)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    with torch.cuda.stream(side):
        got = all_of(z)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    held = torch.zeros_like(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of(held)
    held.copy_(z)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # a row's answers depend on the row alone, to the rounding of how it is aligned
    one = heads.log_probs(z[-1:], y[-1:], top=16, temperature=0.8)
    assert torch.equal(one.index, want[4][-1:])
    within(one.top, f64(want[3][-1:]), 2 ** -16 * (1 + f64(want[3][-1:]).abs()))


def test_rows_beyond_32_bits(dev, heads):
    """Rows more than 2^32 elements into a tensor."""
    c, ld = 100, (1 << 31) + 24
    w = torch.empty(2 * ld + c, dtype=BF16, device=dev)
    z = w.as_strided((3, c), (ld, 1))
    z0, y = logits(dev, BF16, 3, c)
    z.copy_(z0)
    check_answers(heads, z, y, 5)
    check_distill(heads, z, *teacher(dev, z0, 5), None)
    check_gradient(heads, z, y, torch.ones(3, device=dev), None)
    assert torch.equal(z, z0)
    norm = heads.log_probs(z, y).norm
    grad = heads.log_probs_backward(z, norm, y, torch.ones(3, device=dev))
    assert torch.equal(heads.log_probs_backward(z, norm, y, torch.ones(3, device=dev), in_place=True), grad)
    del w


@BOTH
def test_arguments_of_any_kind(dev, heads, dtype):
    """Strided and expanded tensors, numbers of other types, rows of one class."""
    import numpy as np
    z, y = logits(dev, dtype, 6, 300, seed=13)
    want = heads.log_probs(z, y, top=4, temperature=2.0)
    wide = torch.zeros(6, 2, dtype=torch.int32, device=dev)
    wide[:, 1] = y
    got = heads.log_probs(z, wide[:, 1], top=np.int64(4), temperature=torch.tensor(2.0))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g = torch.ones(1, device=dev).expand(6)
    a = heads.log_probs_backward(z, want.norm, y, g, g, temperature=2)
    b = heads.log_probs_backward(z, want.norm.t().contiguous().t(), wide[:, 1], g.contiguous(), g.contiguous(), temperature=2.0)
    assert torch.equal(a, b)
    top, index = teacher(dev, z, 5)
    c = heads.distill(z, top, index, g, temperature=2)
    d = heads.distill(z, top.t().contiguous().t(), index.t().contiguous().t(), g.contiguous(), temperature=2.0)
    assert all(torch.equal(p, q) for p, q in zip(c, d))
    row = z[:1].expand(6, 300)  # one row, six times
    e, f = heads.log_probs(row, y, top=4), heads.log_probs(row.contiguous(), y, top=4)
    assert all(torch.equal(p, q) for p, q in zip(e, f))
    check_answers(heads, z[:, 7:8], torch.zeros(6, dtype=torch.int32, device=dev), 2)
    with pytest.raises(ValueError):
        heads.distill(row, top, index, in_place=True)


def test_refusals(dev, heads):
    from paper_2608_13144_gb300 import LipCacheError
    z, y = logits(dev, F32, 4, 20)
    norm, row = torch.zeros(4, 3, device=dev), torch.zeros(4, device=dev)
    top, index = torch.zeros(4, 3, device=dev), torch.zeros(4, 3, dtype=torch.int32, device=dev)
    for bad in (lambda: heads.log_probs(z.half(), y), lambda: heads.log_probs(z.cpu(), y), lambda: heads.log_probs(z[0], y),
                lambda: heads.log_probs(z, y.long()), lambda: heads.log_probs(z, y[:3]), lambda: heads.log_probs(z, y.cpu()),
                lambda: heads.log_probs(z, y, top=129), lambda: heads.log_probs(z, y, top=-1),
                lambda: heads.log_probs_backward(z, norm[:, :2], y, row),
                lambda: heads.log_probs_backward(z, norm, None, row), lambda: heads.log_probs_backward(z, norm, y, row[:2]),
                lambda: heads.log_probs_backward(z, norm, y, row.bfloat16()),
                lambda: heads.log_probs_backward(z.t()[:, ::2], torch.zeros(20, 3, device=dev), in_place=True),
                lambda: heads.distill(z, top, index[:, :2]), lambda: heads.distill(z, top, index.long()),
                lambda: heads.distill(z, top.bfloat16(), index), lambda: heads.distill(z, top[:, :0], index[:, :0]),
                lambda: heads.distill(z, top, index, row[:3]), lambda: heads.distill(z[:3], top, index),
                lambda: heads.distill(z, top.repeat(1, 50), index.repeat(1, 50)),
                lambda: heads.distill(z.requires_grad_(), top, index), lambda: heads.log_probs(z.requires_grad_(), y),
                lambda: heads.log_probs_backward(z.requires_grad_(), norm, y, row)):
        with pytest.raises(ValueError):
            bad()
    z = z.detach()
    for T in (0.0, -1.0, 1e4, math.nan):
        for bad in (lambda: heads.log_probs(z, y, temperature=T), lambda: heads.distill(z, top, index, temperature=T),
                    lambda: heads.log_probs_backward(z, norm, y, row, temperature=T)):
            with pytest.raises(LipCacheError):
                bad()
    with torch.no_grad():
        heads.log_probs(z.requires_grad_(), y)
