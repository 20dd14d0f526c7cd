"""layer_norm and layer_norm_backward, through the binding, against plain 64-bit
forms on the CPU.

Tolerances, u = 2^-24. Sums of a row go through at most 16 additions of a thread,
5 of its warp and 9 more over warps and blocks, of terms within 3 u of themselves:
within 36 u of their absolute sums. They are taken about a first mean, so that
the row's mean is within its own rounding and 36 u of the mean |x - mean|, the
variance within 80 u and 1 / sqrt within 44 u of themselves.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
BOTH = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
U = 2.0 ** -24


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
    ok = ~nan
    off = (got - want).abs()[ok] - tol.expand_as(want)[ok]
    assert off.numel() == 0 or off.max() <= 0, (what, float(off.max()), int((off > 0).sum()), off.numel())


def case(dev, dtype, n, d, seed=0, offset=0.0):
    gen = torch.Generator().manual_seed(seed + 13 * n + d)
    def rnd(*s):
        return torch.randn(*s, generator=gen)
    x = rnd(n, d) * torch.exp(rnd(1, d)) + rnd(n, 1) + offset
    return x.to(dtype).to(dev), (1 + 0.3 * rnd(d)).to(dev), rnd(d).to(dev), rnd(n, d).to(dtype).to(dev)


def check_norm(heads, x, w, b, eps=1e-5, **kw):
    y, stats = heads.layer_norm(x, w, b, eps=eps, **kw)
    assert y.dtype == x.dtype and stats.dtype == F32
    v, n, d = f64(x), *x.shape
    w = torch.ones(d, dtype=torch.float64) if w is None else f64(w)
    b = torch.zeros(d, dtype=torch.float64) if b is None else f64(b)
    mean = v.mean(1, keepdim=True)
    c = v - mean
    var = c.square().mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    away = c.abs().mean(1, keepdim=True)
    # (the first mean is off by 36 u mean |x|, which its own distances carry on)
    first = 36 * U * v.abs().mean(1, keepdim=True)
    tol_mean = 36 * U * (away + first)
    tol_rstd = (44 * U + 36 * U * first * away / (var + eps)) * rstd
    within(stats[:, :1], mean, tol_mean + U * mean.abs(), "mean")
    within(stats[:, 1:], rstd, tol_rstd, "rstd")
    want = c * rstd * w + b
    tol = w.abs() * (tol_mean * rstd + c.abs() * tol_rstd + 6 * U * (c.abs() + first) * rstd) + 2 * U * want.abs()
    within(y, want, tol + half(x.dtype) * (want.abs() + tol) + 1e-37, "y")
    return y, stats


def check_gradient(heads, dy, x, w, stats, **kw):
    dx, dw, db = heads.layer_norm_backward(dy, x, stats, w, **kw)
    v, g, n, d = f64(x), f64(dy), *x.shape
    wide = torch.ones(d, dtype=torch.float64) if w is None else f64(w)
    rstd = f64(stats)[:, 1:]
    mean = v.mean(1, keepdim=True)  # (the rounded mean's rest is taken out again)
    xh = (v - mean) * rstd
    gw = g * wide
    off = (f64(stats)[:, :1] - mean).abs() * rstd
    tol_x = U * (36 * (xh.abs().mean(1, keepdim=True) + off) + 4 * (xh.abs() + off))
    mg, mgx = gw.mean(1, keepdim=True), (gw * xh).mean(1, keepdim=True)
    tol_mg = 40 * U * gw.abs().mean(1, keepdim=True)
    tol_mgx = 80 * U * (gw.abs() * (xh.abs() + off)).mean(1, keepdim=True) + (gw.abs() * tol_x).mean(1, keepdim=True)
    want = rstd * (gw - mg - xh * mgx)
    tol = rstd * (4 * U * gw.abs() + tol_mg + xh.abs() * tol_mgx + tol_x * mgx.abs() + 4 * U * (mg.abs() + (xh * mgx).abs()))
    if kw.get("need_dx", True):
        assert dx.dtype == x.dtype
        within(dx, want, tol + half(x.dtype) * (want.abs() + tol) + 1e-37, "dx")
    # a column's sum: at most n additions, of terms within tol_x
    if kw.get("need_dweight", True):
        assert dw.dtype == F32
        within(dw, (g * xh).sum(0), (g.abs() * tol_x).sum(0) + (n + 4) * U * (g * xh).abs().sum(0) + 1e-37, "dweight")
    if kw.get("need_dbias", True):
        within(db, g.sum(0), n * U * g.abs().sum(0) + 1e-37, "dbias")
    return dx, dw, db


SIZES = [(1, 1), (1, 2), (2, 3), (5, 8), (3, 17), (40, 64), (33, 200), (70, 256), (9, 257), (1300, 100), (8, 500),
         (300, 512), (5, 513), (4, 1000), (700, 1024), (3, 2047), (6, 2048), (2, 2050), (4, 4096), (400, 4096), (3, 4104),
         (2, 8191), (2, 8192), (2, 8200), (3, 16_384), (2, 16_385), (1, 20_000), (2, 40_000), (1, 65_535), (2, 65_536)]


@BOTH
@pytest.mark.parametrize("n,d", SIZES, ids=lambda v: str(v))
def test_norm(dev, heads, dtype, n, d):
    x, w, b, dy = case(dev, dtype, n, d)
    _, stats = check_norm(heads, x, w, b)
    check_gradient(heads, dy, x, w, stats)
    check_norm(heads, x, None, None, eps=1e-3)
    check_gradient(heads, dy, x, None, stats, need_dx=False)
    check_gradient(heads, dy, x, w, stats, need_dweight=False, need_dbias=False)
    check_gradient(heads, dy, x, w, stats, need_dweight=False)
    check_gradient(heads, dy, x, w, stats, need_dbias=False)


@BOTH
@pytest.mark.parametrize("d", [64, 500, 1000, 5000])
def test_rows_far_from_zero(dev, heads, dtype, d):
    """Features whose mean is far larger than their spread, rows of one value, tiny and large rows."""
    for offset in (100.0, -30_000.0):
        x, w, b, dy = case(dev, dtype, 20, d, offset=offset)
        _, stats = check_norm(heads, x, w, b)
        check_gradient(heads, dy, x, w, stats)
    x[0], x[1], x[2] = 0.0, 1000.0, -3.0
    x[3] *= 1e-20
    x[4] *= 1e8
    _, stats = check_norm(heads, x, w, b, eps=1e-30)
    check_gradient(heads, dy, x, w, stats)
    check_norm(heads, x, w, b, eps=1.0)


@pytest.mark.parametrize("d", [700, 1500, 2050, 4096, 16_385, 20_000, 40_000])
@pytest.mark.parametrize("mean", [1000.1234, 3.3, -30_000.0])
def test_spreads_of_a_few_steps_of_fp32(dev, heads, mean, d):
    """Rows of values a few steps of FP32 above one far from 0, their level other from each 700 columns to the next: the
    row's mean and those of its parts lie between two steps."""
    gen = torch.Generator().manual_seed(d)
    base = torch.tensor(mean, dtype=F32).double()
    step = 2.0 ** (math.floor(math.log2(abs(mean))) - 23)
    steps = torch.randint(0, 3, (5, d), generator=gen) + (torch.arange(d) // 700 * 7 % 4)[None, :]
    exact = base + step * steps
    x = exact.float()
    assert torch.equal(x.double(), exact)
    _, w, b, dy = case(dev, F32, 5, d, seed=1)
    _, stats = check_norm(heads, x.to(dev), w, b, eps=1e-30)
    check_gradient(heads, dy, x.to(dev), w, stats)


@BOTH
@pytest.mark.parametrize("n,d", [(3, 40), (11, 300), (3, 1500), (2, 6000), (2, 9000)])
def test_strides_and_offsets(dev, heads, dtype, n, d):
    x0, w, b, dy0 = case(dev, dtype, n, d, seed=3)
    want, stats = heads.layer_norm(x0, w, b)
    for left, right in ((0, 1), (1, 0), (2, 2), (8, 8), (3, 9)):
        def inside(m):
            t = torch.full((n, left + d + right), math.nan, dtype=dtype, device=dev)
            t[:, left:left + d] = m
            return t[:, left:left + d]
        x, dy = inside(x0), inside(dy0)
        wide = torch.full((n, left + d + right), 7.0, dtype=dtype, device=dev)
        w1 = torch.cat([w[:1], w])[1:]  # off the 16-byte boundary
        check_norm(heads, x, w1, b, out=wide[:, left:left + d])
        assert bool((wide[:, :left] == 7).all()) and bool((wide[:, left + d:] == 7).all())
        check_gradient(heads, dy, x, w1, stats)
    assert torch.equal(heads.layer_norm(x0.t().contiguous().t(), w, b)[0], want)


@BOTH
@pytest.mark.parametrize("d", [100, 900, 9000])
def test_odd_rows_stay_apart(dev, heads, dtype, d):
    x, w, b, dy = case(dev, dtype, 12, d, seed=4)
    clean, stats = heads.layer_norm(x, w, b)
    x[3, 5], x[7, d - 1], x[8, 0] = math.nan, math.inf, -math.inf
    y, s = heads.layer_norm(x, w, b)
    odd = torch.tensor([3, 7, 8], device=dev)
    assert torch.isnan(y[odd]).all() and torch.isnan(s[odd, 1]).all()
    keep = torch.ones(12, dtype=torch.bool, device=dev)
    keep[odd] = False
    assert torch.equal(y[keep], clean[keep]) and torch.equal(s[keep], stats[keep])
    dx = heads.layer_norm_backward(dy, x, s, w)[0]
    assert torch.isnan(dx[odd]).all() and torch.isfinite(dx[keep]).all()


@BOTH
def test_gradient_against_differences(dev, heads, dtype):
    n, d, eps = 5, 90, 1e-5
    x, w, b, dy = case(dev, dtype, n, d, seed=6)
    _, stats = heads.layer_norm(x, w, b, eps=eps)
    grads = heads.layer_norm_backward(dy, x, stats, w)
    gen = torch.Generator().manual_seed(2)

    def f(x, w, b):
        c = x - x.mean(1, keepdim=True)
        return float((f64(dy) * (c / torch.sqrt(c.square().mean(1, keepdim=True) + eps) * w + b)).sum())

    at = [f64(x), f64(w), f64(b)]
    for i, g in enumerate(grads):
        step = torch.randn(at[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + 1e-5 * step, at[i] - 1e-5 * step
        diff = (f(*up) - f(*down)) / 2e-5
        # the outputs' rounding (of dweight and dbias: FP32's), 2^-17 of their own terms, the differences' 1e-6
        size = float((f64(g).abs() * step.abs()).sum())
        assert abs(diff - float((f64(g) * step).sum())) <= (half(g.dtype) + 2 ** -17) * size + 1e-6 * (1 + size), i


@BOTH
@pytest.mark.parametrize("n,d", [(3000, 256), (900, 4096), (50, 20_000)])
def test_repeats_on_streams_and_in_graphs(dev, heads, dtype, n, d):
    x, w, b, dy = case(dev, dtype, n, d, seed=7)

    def all_of(x):
        y, stats = heads.layer_norm(x, w, b)
        return (y, stats, *heads.layer_norm_backward(dy, x, stats, w))

    want = all_of(x)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(want, all_of(x)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    with torch.cuda.stream(side):
        got = all_of(x)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    held = torch.ones_like(x)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    got = []
    for g in graphs:  # two graphs, each with a workspace of its own
        with torch.cuda.graph(g):
            got.append(all_of(held))
    held.copy_(x)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    for one in got:
        assert all(torch.equal(p, q) for p, q in zip(want, one))
    # a row's result depends on the row alone
    assert torch.equal(heads.layer_norm(x[-1:], w, b)[0], want[0][-1:])


@BOTH
def test_empty_batches(dev, heads, dtype):
    x = torch.empty(0, 40, dtype=dtype, device=dev)
    y, stats = heads.layer_norm(x)
    assert y.shape == (0, 40) and stats.shape == (0, 2)
    dx, dw, db = heads.layer_norm_backward(x, x, stats)
    assert dx.shape == (0, 40) and not dw.any() and not db.any() and dw.shape == db.shape == (40,)


def test_rows_beyond_32_bits(dev, heads):
    d, ld = 64, (1 << 31) + 24
    t = torch.empty(2 * ld + d, dtype=BF16, device=dev)
    x = t.as_strided((3, d), (ld, 1))
    x0, w, b, dy = case(dev, BF16, 3, d)
    x.copy_(x0)
    (y, s), (y0, s0) = heads.layer_norm(x, w, b), heads.layer_norm(x0, w, b)
    assert torch.equal(y, y0) and torch.equal(s, s0)
    for p, q in zip(heads.layer_norm_backward(dy, x, s, w), heads.layer_norm_backward(dy, x0, s, w)):
        assert torch.equal(p, q)
    del t


def test_refusals(dev, heads):
    from paper_2608_13144_gb300 import LipCacheError
    x, w, b, dy = case(dev, F32, 4, 20)
    _, stats = heads.layer_norm(x)
    for bad in (lambda: heads.layer_norm(x.half()), lambda: heads.layer_norm(x.cpu()), lambda: heads.layer_norm(x[0]),
                lambda: heads.layer_norm(x, w[:3]), lambda: heads.layer_norm(x, w.bfloat16()),
                lambda: heads.layer_norm(x, w, b.cpu()), lambda: heads.layer_norm(x, out=dy.bfloat16()),
                lambda: heads.layer_norm(x, out=dy[:3]), lambda: heads.layer_norm(x.t(), out=dy.t()),
                lambda: heads.layer_norm_backward(dy.bfloat16(), x, stats), lambda: heads.layer_norm_backward(dy[:3], x, stats),
                lambda: heads.layer_norm_backward(dy, x, stats[:, :1]), lambda: heads.layer_norm_backward(dy, x, stats, w[:2]),
                lambda: heads.layer_norm(x.requires_grad_()), lambda: heads.layer_norm(x.detach(), w.requires_grad_()),
                lambda: heads.layer_norm_backward(dy.requires_grad_(), x.detach(), stats)):
        with pytest.raises(ValueError):
            bad()
    x = x.detach()
    for eps in (0.0, -1.0, 2.0, math.nan):
        with pytest.raises(LipCacheError):
            heads.layer_norm(x, eps=eps)
    wide = torch.empty(1, 65_537, device=dev)
    for bad in (lambda: heads.layer_norm(wide), lambda: heads.layer_norm_backward(wide, wide, stats[:1])):
        with pytest.raises(LipCacheError):
            bad()
    out = torch.empty_like(x)
    version = out._version
    heads.layer_norm(x, out=out)
    assert out._version > version
