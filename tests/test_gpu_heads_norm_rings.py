"""Layer norm and its gradients where each group of threads takes many rows, so that
rows come through the places of its ring of asynchronous copies again and again: the
64-bit forms and tolerances of test_gpu_heads_norm.py, on the GPU.

How many groups the device holds goes by registers and shared memory; the sizes are
for 152 SMs, whose groups take nine rows each at the least (a ring is three or four
deep): aligned rows and others, of one warp, several warps and a cluster.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_gpu_heads_norm as plain  # noqa: E402
from test_gpu_heads_norm import BOTH, dev, heads  # noqa: E402,F401

SIZES = [(100_000, 96), (100_000, 100), (100_001, 101), (70_000, 257), (70_000, 384), (40_000, 1000), (40_001, 1001),
         (20_000, 2047), (20_000, 2048), (10_000, 4001), (10_000, 4096), (5000, 8000), (5000, 8191), (1600, 16_383),
         (1600, 16_384), (1000, 20_000), (1000, 20_001), (500, 40_000), (500, 40_001)]


def case(dev, dtype, n, d):
    gen = torch.Generator(device=dev).manual_seed(n + d)

    def rnd(*s):
        return torch.randn(*s, generator=gen, device=dev)

    x = rnd(n, d) * torch.exp(rnd(1, d)) + rnd(n, 1)
    return x.to(dtype), 1 + 0.3 * rnd(d), rnd(d), rnd(n, d).to(dtype)


@BOTH
@pytest.mark.parametrize("n,d", SIZES, ids=lambda v: str(v))
def test_many_rows_a_group(dev, heads, dtype, n, d, monkeypatch):
    monkeypatch.setattr(plain, "f64", lambda t: t.detach().double())
    x, w, b, dy = case(dev, dtype, n, d)
    y, stats = plain.check_norm(heads, x, w, b)
    grads = plain.check_gradient(heads, dy, x, w, stats)
    # without dx rows are only read; a second pass finds the rings as the first one left them
    _, dw, db = heads.layer_norm_backward(dy, x, stats, w, need_dx=False)
    assert torch.equal(dw, grads[1]) and torch.equal(db, grads[2])
    again = heads.layer_norm(x, w, b)
    assert torch.equal(again[0], y) and torch.equal(again[1], stats)


@BOTH
@pytest.mark.parametrize("n,d", [(60_000, 200), (20_000, 1500), (1000, 20_000)])
def test_many_rows_a_group_at_any_stride(dev, heads, dtype, n, d, monkeypatch):
    """Rows inside wider ones: each at another offset from the 16-byte boundaries, what stands beside them untouched."""
    monkeypatch.setattr(plain, "f64", lambda t: t.detach().double())
    x0, w, b, dy0 = case(dev, dtype, n, d)
    wide = torch.full((n, d + 5), float("nan"), dtype=dtype, device=dev)
    x = wide[:, 3:3 + d]
    x.copy_(x0)
    dy = torch.full((n, d + 2), float("nan"), dtype=dtype, device=dev)[:, 1:1 + d]
    dy.copy_(dy0)
    out = torch.full((n, d + 1), 7.0, dtype=dtype, device=dev)
    _, stats = plain.check_norm(heads, x, w, b, out=out[:, 1:])
    assert bool((out[:, 0] == 7).all())
    plain.check_gradient(heads, dy, x, w, stats)
