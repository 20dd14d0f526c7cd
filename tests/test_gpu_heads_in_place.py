"""Gradients written over the logits: log_probs_backward and distill in place give
what they give in an array of their own, bit for bit, on each way that a row can take
(a few lanes, a block with the row in registers or shared memory, a cluster, rows read
twice from memory), and touch nothing beside their rows.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_heads_answers import BOTH, check_distill, check_gradient, dev, heads, logits, teacher  # noqa: E402,F401

SIZES = [(500, 30), (500, 100), (500, 200), (300, 1000), (40, 3000), (40, 12_345), (40, 30_000), (20, 50_001), (40, 50_001),
         (33, 140_001), (2, 400_003), (2, 460_003)]


@BOTH
@pytest.mark.parametrize("n,c", SIZES, ids=lambda v: str(v))
def test_in_place(dev, heads, dtype, n, c):
    z0, y = logits(dev, dtype, n, c, seed=20)
    gen = torch.Generator().manual_seed(c)
    g, h = torch.randn(n, generator=gen).to(dev), torch.randn(n, generator=gen).to(dev)
    top, index = teacher(dev, z0, 20)
    index[n // 2, 1] = index[n // 2, 0]  # a class named twice
    w = torch.rand(n, generator=gen).to(dev)
    policy = check_gradient(heads, z0, y, g, h, 0.7)
    _, student = check_distill(heads, z0, top, index, w, 2.0)
    norm = heads.log_probs(z0, y, temperature=0.7).norm

    for left, right in ((0, 0), (8, 8), (0, 3), (5, 2)):
        wide = torch.full((n, left + c + right), math.nan, dtype=dtype, device=dev)
        z = wide[:, left:left + c]
        for at, call in enumerate((lambda: heads.log_probs_backward(z, norm, y, g, h, temperature=0.7, in_place=True),
                                   lambda: heads.distill(z, top, index, w, temperature=2.0, in_place=True)[1])):
            z.copy_(z0)
            apart = (heads.log_probs_backward(z, norm, y, g, h, temperature=0.7) if at == 0
                     else heads.distill(z, top, index, w, temperature=2.0)[1])
            if left == right == 0:
                assert torch.equal(apart, (policy, student)[at])
            got = call()
            assert got.data_ptr() == z.data_ptr()
            assert torch.equal(z, apart)
            assert torch.isnan(wide[:, :left]).all() and torch.isnan(wide[:, left + c:]).all()
