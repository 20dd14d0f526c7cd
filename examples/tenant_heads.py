"""Train several tenants' heads over one shared head, then certify and serve them.

Every tenant labels the same features in its own way: some classes trade
places. A tenant's head is the shared one plus a low-rank adapter,
W + s_g B_g A_g. Each training step takes a batch with all tenants' rows mixed
(logits, losses with their gradient, the adapters' gradients, the optimiser's
step), at once for all tenants. Then each tenant's head is merged and certified
in a cache of its own; queries are answered from the caches, and those that
miss by the heads themselves, one call for all tenants.

    python examples/tenant_heads.py [--tenants 4] [--steps 100]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_13144_gb300 import heads  # noqa: E402
from paper_2608_13144_gb300.lipcache import LipCache  # noqa: E402


def features(centres: torch.Tensor, n: int, noise: float, rng: torch.Generator):
    """n rows around the classes' centres, and their classes."""
    label = torch.randint(centres.shape[0], (n,), generator=rng, device=centres.device)
    x = centres[label] + noise * torch.randn(n, centres.shape[1], generator=rng, device=centres.device)
    return x, label


def run(tenants: int = 4, classes: int = 20, d: int = 96, rank: int = 8, steps: int = 100, batch: int = 1024,
        rows: int = 4096, queries: int = 2048, lr: float = 0.05, seed: int = 0, device: str = "cuda:0") -> dict:
    rng = torch.Generator(device).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=rng, device=device)

    # The shared head: the nearest centre's class.
    centres = torch.nn.functional.normalize(normal(classes, d), dim=1)
    W, bias = 8 * centres, torch.zeros(classes, device=device)
    # A tenant's labels: `rank` of the classes move on by one place.
    relabel = torch.arange(classes, device=device).repeat(tenants, 1)
    for g in range(tenants):
        moved = torch.randperm(classes, generator=rng, device=device)[:rank]
        relabel[g, moved] = moved.roll(1)

    A, B = normal(tenants, rank, d) / d ** 0.5, torch.zeros(tenants, classes, rank, device=device)
    momentum_A, momentum_B = torch.zeros_like(A), torch.zeros_like(B)
    scales = torch.full((tenants,), 2.0, device=device)
    weight = torch.full((batch,), 1.0 / batch, device=device)

    def accuracy():
        x, label = features(centres, queries, 0.05, rng)
        g = torch.randint(tenants, (queries,), generator=rng, device=device, dtype=torch.int32)
        y = heads.adapted_logits(x, W, A, B, g, bias, scales)
        return (y.argmax(1) == relabel[g.long(), label]).float().mean().item()

    report = {"accuracy_before": accuracy(), "loss": []}
    for step in range(steps):
        x, label = features(centres, batch, 0.05, rng)
        g = torch.randint(tenants, (batch,), generator=rng, device=device, dtype=torch.int32)
        target = relabel[g.long(), label].int()
        logits = heads.adapted_logits(x, W, A, B, g, bias, scales)
        loss, dlogits = heads.cross_entropy(logits, target, weight, in_place=True)
        _, dA, dB = heads.adapted_logits_backward(dlogits, x, W, A, B, g, scales, need_dx=False)
        now = lr * (1 - step / steps)
        heads.orthogonal_step(A, dA, momentum_A, now)
        heads.orthogonal_step(B, dB, momentum_B, now)
        report["loss"].append(loss.sum())
    report["loss"] = torch.stack(report["loss"]).tolist()
    report["accuracy_after"] = accuracy()

    # Serving: a cache per tenant, certified for its merged head; the queries
    # that no cache answers go to the heads together.
    answered, left, left_tenant, left_slot = [], [], [], []
    merged = W + scales[:, None, None] * torch.bmm(B, A)
    for g in range(tenants):
        keys, _ = features(centres, rows, 0.05, rng)
        with LipCache(d, classes, rows, device=torch.device(device)) as cache:
            cache.set_head(merged[g].contiguous(), bias)
            cache.insert(keys)
            near = keys[torch.randint(rows, (queries // 2,), generator=rng, device=device)]
            near = near + 0.002 * normal(queries // 2, d)
            fresh, _ = features(centres, queries - queries // 2, 0.05, rng)
            q = torch.cat([near, fresh])
            hit, label, _ = cache.probe(q)
        answered.append((q, hit, label))
        miss = (hit < 0).nonzero().flatten()
        left.append(q[miss])
        left_tenant.append(torch.full((len(miss),), g, dtype=torch.int32, device=device))
        left_slot.append(miss)
    fallback = heads.adapted_logits(torch.cat(left), W, A, B, torch.cat(left_tenant), bias, scales).argmax(1).int()
    for (q, hit, label), miss, own in zip(answered, left_slot, fallback.split([len(m) for m in left_slot])):
        label[miss] = own

    # What a cache answered is what the tenant's own head would have.
    hits = agree = 0
    for g, (q, hit, label) in enumerate(answered):
        own = heads.adapted_logits(q, W, A, B, torch.full((queries,), g, dtype=torch.int32, device=device), bias,
                                   scales).argmax(1)
        hits += int((hit >= 0).sum())
        agree += int((own[hit >= 0] == label[hit >= 0]).sum())
    report["hit_rate"] = hits / (tenants * queries)
    report["hits_agree"] = agree / max(hits, 1)
    report["answered"] = all(bool((label >= 0).all()) for _, _, label in answered)
    return report


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tenants", type=int, default=4)
    ap.add_argument("--steps", type=int, default=100)
    a = ap.parse_args()
    r = run(tenants=a.tenants, steps=a.steps)
    print(f"loss {r['loss'][0]:.3f} -> {r['loss'][-1]:.3f}, accuracy {r['accuracy_before']:.3f} -> "
          f"{r['accuracy_after']:.3f}; {100 * r['hit_rate']:.1f}% of the queries answered by the caches, "
          f"{100 * r['hits_agree']:.1f}% of those as the tenant's own head answers")


if __name__ == "__main__":
    main()
