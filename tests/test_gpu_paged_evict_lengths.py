"""Eviction that writes the new lengths over the old ones, which its other CTAs read."""
from __future__ import annotations

import pytest
import torch

from .test_gpu_paged import handle, pkg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hkv,budget,extra", [(40, 8, 512, 90), (3, 2, 2048, 1), (64, 1, 9, 300), (16, 8, 700, 0)])
def test_lengths_over_the_source_as_into_their_own(pkg, B, Hkv, budget, extra):  # noqa: F811
    """Many CTAs behind the one that sets the lengths, again and again: the rows, slots and weights of a call with lengths of their own."""
    g, D, page = torch.Generator(device="cuda").manual_seed(B), 64, 16
    lens = torch.randint(max(1, budget - 50), budget + extra + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    pages, to = -(-(budget + extra) // page), -(-budget // page)
    n = B * (pages + to)
    perm = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(B, -1)
    table, table_to = perm[:, :pages].contiguous(), perm[:, pages:].contiguous()
    k, v = (torch.randn(n, Hkv, page, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(n, Hkv, page, generator=g, device="cuda")
    h = handle(pkg, Hkv, Hkv, D, "bf16", page_size=page, max_batch=B, max_pages=pages)

    def evict(aliased):
        pool, src = [t.clone() for t in (k, v, w)], lens.clone()
        dst = src if aliased else torch.zeros_like(lens)
        kept = torch.empty(B, Hkv, budget, dtype=torch.int32, device="cuda")
        h.evict(h.cache(*pool[:2], table, src, weights=pool[2]), h.cache(*pool[:2], table_to, dst, weights=pool[2]), kept, sinks=2, recent=3)
        return [*pool, kept, dst]

    want = evict(False)
    assert torch.equal(want[4], lens.clamp(max=budget))
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(evict(True), want))
    assert h.status() == 0
    h.close()
