"""The window example: a ring of pages holds what attention sees, for sequences far
longer than the pool."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

from . import codes_ref as ref
from .paged_ref import within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("window,sinks", [(32, 4), (45, 0), (33, 20)])
def test_example_sees_its_window(cache, window, sinks):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "window_decode.py")
    spec = importlib.util.spec_from_file_location("window_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    B, hidden, D = 2, 128, 64
    layer = example.Layer(B, window, sinks, 400, cache=cache, hidden=hidden, n_q_heads=8, n_kv_heads=2, head_dim=D, page=16)
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda n: torch.randn(B, n, hidden, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    layer.prompt(rand(30), torch.tensor([30, 7], dtype=torch.int32, device="cuda"))
    rows = {b: {} for b in range(B)}     # what each slot's value was when it was written, by the formula
    for token in range(300):
        layer.x.copy_(rand(1))
        lens = layer.kv_len.tolist()
        _, _, v = layer.rows(layer.x)
        layer.step()
        for b in range(B):
            rows[b][lens[b]] = v[b, 0].double().cpu()
        if token % 37 and token < 298:
            continue
        now = layer.kv_len.tolist()
        assert now == [n + 1 for n in lens]
        kv, vv = ref.values(layer.k_pages, layer.k_scales), ref.values(layer.v_pages, layer.v_scales)
        o, _, _, to, _, _ = ref.attend(layer.q_out.view(B, 8, D), kv, vv, layer.cache.block_table, now, D ** -0.5, window, sinks,
                                       layer.v_scales.cpu())
        within(layer.out.cpu(), o, to, f"token {token}")
        table = layer.cache.block_table.cpu().long()
        for b in range(B):
            for j in ref.seen(now[b], window, sinks).tolist():
                if j in rows[b]:         # the ring still holds the row that was stored there, not a later one
                    got, x = vv[table[b, j // 16], :, j % 16], rows[b][j]
                    s = layer.v_scales[table[b, j // 16], :, 0].cpu().double()[:, None]
                    assert ((got - x).abs() <= (2.0 ** -4 * x.abs() + 2.0 ** -9 * s if cache == "e4m3" else s)).all(), (token, b, j)
    assert layer.att.status() == 0
    with pytest.raises(ValueError):
        layer.prompt(rand(400), None)
    layer.att.close()
