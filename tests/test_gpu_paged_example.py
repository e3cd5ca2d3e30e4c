"""The decode example counts every token's attention weights once."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

from . import paged_ref as ref

pytestmark = pytest.mark.gpu


def test_example_accumulates_each_token_once():
    """A token adds its heads' probabilities, one unit each, to the rows of its KV head: also the first one after a graph
    was captured, in either half of the pool."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    B, hidden, prompt, budget = 2, 128, 40, 30
    layer = example.Layer(B, budget, 20, 200, hidden=hidden, n_q_heads=8, n_kv_heads=2, sinks=2, recent=8)
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda n: torch.randn(B, n, hidden, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    layer.prompt(rand(prompt), torch.tensor([prompt, 33], dtype=torch.int32, device="cuda"))

    def held():
        cache = layer.caches[layer.at]
        return torch.stack([ref.gather(layer.weights, cache.block_table[b].cpu(), int(layer.kv_len[b])).sum(1) for b in range(B)])

    for half in range(2):
        was = held()
        for token in range(3):
            layer.x.copy_(rand(1))
            layer.step()
            # 4 query heads to a KV head; weights are fp32 sums of some 50 rows
            assert (held() - was - 4 * (token + 1)).abs().max() < 1e-4, (half, token)
        layer.evict()
    assert layer.pos.tolist() == [prompt + 6, 33 + 6] and layer.att.status() == 0
    layer.att.close()
