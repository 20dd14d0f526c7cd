"""The operators that train and serve heads at the sizes where they take another
path than small ones do: tiles of CTA pairs, a launch a product, several tiles
a CTA, joined parts. Same 64-bit forms and tolerances as test_gpu_heads.py.

Which path a size takes depends on the number of SMs; the sizes are for 152.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_heads import BF16, F32, QUINTIC, UNIT, check_ortho, dev, f64, heads, ortho_exact, within  # noqa: E402,F401


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
