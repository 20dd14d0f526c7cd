"""The operators that train and serve heads at the sizes where they take another
path than small ones do: tiles of CTA pairs, a launch a product, several tiles
a CTA, joined parts. Same 64-bit forms and tolerances as test_gpu_heads.py.

Which path a size takes depends on the number of SMs; the sizes are for 152.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_heads import (  # noqa: E402,F401
    BF16, F32, POLAR, QUINTIC, UNIT, adapted_case, adapted_exact, check_ortho, dev, f64, heads, ortho_exact, tolerance,
    within)


# ---------------------------------------------------------------- several tiles a CTA
# batch, rows, cols: more than 2 x 152 tiles of 128 columns in the update, rows that leave a tile's last quarters empty
MANY_TILES = [(40, 96, 2048), (33, 72, 2049), (70, 65, 700), (6, 190, 4003), (1, 24, 65_536), (2, 30, 40_001),
              (24, 2500, 66), (3, 20_001, 100)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,m,n", MANY_TILES)
def test_orthogonalize_many_tiles_a_cta(dev, heads, dtype, batch, m, n):
    """Warps of the epilogue that have nothing to write run ahead of those
    that have; each reads its own tile's X."""
    gen = torch.Generator().manual_seed(batch + m)
    g = torch.randn(batch, m, n, generator=gen).to(dtype)
    got = heads.orthogonalize(g.to(dev), steps=3)
    for i in range(batch):
        check_ortho(heads, got[i], g[i].double(), dtype, 3, QUINTIC)
    assert torch.equal(heads.orthogonalize(g.to(dev), steps=3), got)


@pytest.mark.parametrize("batch,m,n", [(40, 96, 2048), (33, 72, 2049), (24, 2500, 66)])
def test_orthogonal_step_many_tiles_a_cta(dev, heads, batch, m, n):
    gen = torch.Generator().manual_seed(batch + n)
    grad, mom, w = (torch.randn(batch, m, n, generator=gen) for _ in range(3))
    grad, w = grad.to(BF16), (w / math.sqrt(n)).to(BF16)
    ow, om = heads.orthogonal_step(w.to(dev), grad.to(dev), mom.to(dev), 0.3, 0.9, True, 0.1, steps=3)
    new = 0.9 * mom.double() + 0.1 * grad.double()
    d = 0.9 * new + 0.1 * grad.double()
    within(om, new, 4 * UNIT[F32] * (mom.double().abs() + grad.double().abs()))
    keep, rate = 1 - 0.3 * 0.1, 0.3 * math.sqrt(max(1.0, m / n))
    for i in range(batch):
        o = ortho_exact(d[i], 3, QUINTIC, 1e-7)
        noise = max(float(torch.linalg.vector_norm(ortho_exact(d[i], 3, QUINTIC, 1e-7, 2.0 ** -11, k) - o)) for k in range(3))
        want = keep * w[i].double() - rate * o
        off = float(torch.linalg.vector_norm(f64(ow[i]) - want))
        assert off <= 8 * rate * noise + 2 * UNIT[BF16] * float(torch.linalg.vector_norm(want)) + 1e-6 * rate, i


# ---------------------------------------------------------------- a launch a product
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,m,n", [(5, 1030, 1100), (5, 1101, 1030), (3, 1290, 1801), (20, 520, 512)])
def test_orthogonalize_large(dev, heads, dtype, batch, m, n):
    """Tiles of CTA pairs: the triangles of S and P, their mirror images, ragged edges, several matrices."""
    gen = torch.Generator().manual_seed(batch + m)
    g = torch.randn(batch, m, n, generator=gen).to(dtype)
    got = heads.orthogonalize(g.to(dev), steps=3, coefficients=[QUINTIC, POLAR, QUINTIC])
    for i in (0, batch // 2, batch - 1):
        check_ortho(heads, got[i], g[i].double(), dtype, 3, [QUINTIC, POLAR, QUINTIC])
    assert torch.equal(heads.orthogonalize(g.to(dev), steps=3, coefficients=[QUINTIC, POLAR, QUINTIC]), got)


@pytest.mark.parametrize("wt,gt", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)],
                         ids=["f32", "bf16", "bf16_f32", "f32_bf16"])
@pytest.mark.parametrize("batch,m,n", [(5, 1030, 1104), (5, 1101, 1030)])
def test_orthogonal_step_large(dev, heads, wt, gt, batch, m, n):
    gen = torch.Generator().manual_seed(m)
    grad, mom, w = (torch.randn(batch, m, n, generator=gen) for _ in range(3))
    grad, w = grad.to(gt), (w / math.sqrt(n)).to(wt)
    W, M = w.to(dev), mom.to(dev)
    heads.orthogonal_step(W, grad.to(dev), M, 0.3, 0.9, True, 0.1, steps=3)
    new = 0.9 * mom.double() + 0.1 * grad.double()
    within(M, new, 4 * UNIT[F32] * (mom.double().abs() + grad.double().abs()))
    keep, rate = 1 - 0.3 * 0.1, 0.3 * math.sqrt(max(1.0, m / n))
    for i in (0, batch - 1):
        d = 0.9 * new[i] + 0.1 * grad[i].double()
        o = ortho_exact(d, 3, QUINTIC, 1e-7)
        unit = 2.0 ** (-21 if wt == F32 else -11)
        noise = max(float(torch.linalg.vector_norm(ortho_exact(d, 3, QUINTIC, 1e-7, unit, k) - o)) for k in range(3))
        want = keep * w[i].double() - rate * o
        off = float(torch.linalg.vector_norm(f64(W[i]) - want))
        assert off <= 8 * rate * noise + 2 * UNIT[wt] * float(torch.linalg.vector_norm(want)) + 1e-6 * rate, i


# ---------------------------------------------------------------- tiles of CTA pairs
PAIRS = [
    # n, d, c, g, r, ids: 38 tiles of 256 x 256 and more, of the logits or of the features' gradient
    (2500, 200, 1100, 3, 16, "mixed"), (2500, 200, 1100, 40, 16, "mixed"), (2500, 200, 1100, 12, 16, "grouped"),
    (2500, 1100, 200, 5, 40, "mixed"), (2500, 1100, 200, 60, 8, "mixed"), (2500, 1105, 1300, 1, 128, "one"),
    (2500, 1100, 1101, 3, 5, "none"), (5000, 520, 1032, 2, 64, "mixed"), (5001, 72, 513, 2, 100, "grouped"),
    (20_000, 64, 520, 4, 8, "mixed"), (20_001, 260, 40, 17, 16, "mixed"), (10_000, 100, 264, 300, 2, "mixed"),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", PAIRS, ids=lambda s: "x".join(map(str, s)))
def test_adapted_large(dev, heads, dtype, shape):
    """Pairs' lane masks, drained sums, dense low-rank stages and operands contracted over their rows; rows of FP32
    factors in groups of 32 and 128 a block; outer products over clusters and windows of rows."""
    n, d, c, g, r, ids = shape
    t, a, s, bias = adapted_case(dev, dtype, n, d, c, g, r, ids, seed=21)
    (y, dx, dA, dB), (ty, tdx, tdA, tdB) = adapted_exact(t, a, s, bias)
    got = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s)
    within(got, y, tolerance(dtype, y, ty, d + r), "y")
    gx, gA, gB = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)
    within(gx, dx, tolerance(dtype, dx, tdx, c + r), "dx")
    within(gA, dA, tolerance(dtype, dA, tdA, c + n), "dA")
    within(gB, dB, tolerance(dtype, dB, tdB, d + n), "dB")
    again = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s)
    assert all(torch.equal(p, q) for p, q in zip((gx, gA, gB), again))
    assert torch.equal(got, heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,c,g,r", [(640, 256, 192, 5, 16), (2500, 200, 1100, 40, 16), (2500, 200, 1100, 3, 8)])
def test_adapted_order_of_rows_within_rounding(dev, heads, dtype, n, d, c, g, r):
    """Rows in another order: the sums' terms are the same, their order may not be."""
    t, a, s, bias = adapted_case(dev, dtype, n, d, c, g, r, "mixed", seed=4)
    (y, *_), (terms, *_) = adapted_exact(t, a, s, bias)
    one = heads.adapted_logits(t["x"], t["W"], t["A"], t["B"], a, bias=bias, scales=s)
    at = torch.argsort(a, stable=True)
    two = heads.adapted_logits(t["x"][at], t["W"], t["A"], t["B"], a[at], bias=bias, scales=s)
    within(two, f64(one)[at.cpu()], 2 * tolerance(dtype, y, terms, d + r)[at.cpu()])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,c,g,r", [(1, 40, 30, 2, 4), (300, 248, 520, 6, 8), (2500, 1100, 200, 40, 8)])
def test_adapted_gradients_one_at_a_time(dev, heads, dtype, n, d, c, g, r):
    """Each gradient is right whether or not the others are asked for (the parts of a sum may differ)."""
    t, a, s, _ = adapted_case(dev, dtype, n, d, c, g, r, "mixed", seed=31)
    (_, *want), (_, *terms) = adapted_exact(t, a, s, None)
    for mask in range(8):
        need = [bool(mask & 1), bool(mask & 2), bool(mask & 4)]
        got = heads.adapted_logits_backward(t["dy"], t["x"], t["W"], t["A"], t["B"], a, scales=s, need_dx=need[0],
                                            need_dA=need[1], need_dB=need[2])
        for k, K in enumerate((c + r, c + n, d + n)):
            if need[k]:
                within(got[k], want[k], tolerance(dtype, want[k], terms[k], K), f"{k} of {need}")
            else:
                assert got[k] is None


# ---------------------------------------------------------------- graphs
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,c", [(1, 256, 200), (48, 264, 520), (700, 256, 200), (2500, 200, 1100)])
def test_head_operators_in_a_graph(dev, heads, dtype, n, d, c):
    """A training step captured once and replayed on other rows does what the calls do."""
    t, a, s, bias = adapted_case(dev, dtype, n, d, c, 5, 8, "mixed", seed=41)
    gen = torch.Generator().manual_seed(n)
    target = torch.randint(0, c, (n,), generator=gen).to(torch.int32).to(dev)

    def step(x, ids, y):
        z = heads.adapted_logits(x, t["W"], t["A"], t["B"], ids, bias=bias, scales=s)
        loss, dz = heads.cross_entropy(z, y)
        return (z, loss, dz, *heads.adapted_logits_backward(dz, x, t["W"], t["A"], t["B"], ids, scales=s))

    x, ids, y = t["x"].clone(), a.clone(), target.clone()
    step(x, ids, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, ids, y)
    for shift in (1, 3):
        x.copy_(t["x"].roll(shift, 1))
        ids.copy_(a.roll(shift, 0))
        y.copy_(target.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        want = step(x, ids, y)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,m,n", [(3, 16, 200), (1, 200, 256), (2, 333, 140), (5, 1030, 1100)])
def test_orthogonalisation_in_a_graph(dev, heads, dtype, batch, m, n):
    gen = torch.Generator().manual_seed(n)
    g, h = (torch.randn(batch, m, n, generator=gen).to(dtype).to(dev) for _ in range(2))
    w, mom = torch.randn(batch, m, n, generator=gen).to(dtype).to(dev), torch.randn(batch, m, n, generator=gen).to(dev)
    want_o = heads.orthogonalize(h, steps=3)
    want = heads.orthogonal_step(w, h, mom, 0.1, steps=3, out=(torch.empty_like(w), torch.empty_like(mom)))
    torch.cuda.synchronize()
    x, out = g.clone(), (torch.empty_like(w), torch.empty_like(mom))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = heads.orthogonalize(x, steps=3)
        heads.orthogonal_step(w, x, mom, 0.1, steps=3, out=out)
    x.copy_(h)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want_o) and all(torch.equal(p, q) for p, q in zip(out, want))
