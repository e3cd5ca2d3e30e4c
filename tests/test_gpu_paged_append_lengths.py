"""Append where a sequence's length is outside its block table: no row of it is stored."""
from __future__ import annotations

import pytest
import torch

from . import paged_ref as ref
from .test_gpu_paged import DT, EPS, bf16_more, handle, pkg, rows_case  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [-2, -1, -2 ** 31, 33, 2 ** 31 - 1])
def test_append_to_a_length_outside_the_table(pkg, dtype, length):  # noqa: F811
    """Five new rows: those past slot -1 would otherwise go to the sequence's first slots."""
    B, n, H, D, page = 3, 5, 4, 64, 16
    q, k, v, g_q, g_k, _, _, rope = rows_case(pkg, Hq=H, Hkv=H, D=D, dtype=dtype, B=B, n=n, gains=True)
    h = handle(pkg, H, H, D, dtype, page_size=page, max_batch=B, max_pages=2)
    g = torch.Generator(device="cuda").manual_seed(1)
    kp, vp = (torch.randn(6, H, page, D, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    w = torch.rand(6, H, page, generator=g, device="cuda")
    table = torch.tensor([[5, 1], [0, 2], [4, 3]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([7, length, 0], dtype=torch.int32, device="cuda")
    pos = torch.tensor([7, 3, 0], dtype=torch.int32, device="cuda")
    before = [t.clone() for t in (kp, vp, w)]
    qo = torch.empty(B, n, H, D, dtype=DT[dtype], device="cuda")
    h.append(h.cache(kp, vp, table, kv_len, weights=w), q, k, v, qo, rope, g_q=g_q, g_k=g_k, pos=pos)
    assert h.status() == 2
    for t, was in zip((kp, vp, w), before):
        assert torch.equal(t[[0, 2]], was[[0, 2]])                # the sequence's pages are as they were
        assert not torch.equal(t[[5, 4]], was[[5, 4]])
    for b in range(B):                                              # queries of every sequence, keys of the others
        y, tol = ref.norm_rope(q[b], g_q, rope, int(pos[b]), EPS)
        ref.within(qo[b], y, tol + bf16_more(dtype, y), "q")
    for b, slot in ((0, 7), (2, 0)):
        y, tol = ref.norm_rope(k[b], g_k, rope, int(pos[b]), EPS)
        ref.within(kp[int(table[b, 0]), :, slot:slot + n].transpose(0, 1), y, tol + bf16_more(dtype, y), "k")
        assert torch.equal(vp[int(table[b, 0]), :, slot:slot + n].transpose(0, 1), v[b])
        assert (w[int(table[b, 0]), :, slot:slot + n] == 0).all()
    h.close()
