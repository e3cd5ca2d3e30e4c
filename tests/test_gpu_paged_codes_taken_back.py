"""Rows that are taken back: a draft's rows are appended, and the length goes back to the
rows that were accepted.  Their block keeps the scale that it had with the others."""
from __future__ import annotations

import pytest
import torch

from . import codes_ref as ref
from .test_gpu_paged_codes import append_case, identity_rope, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D,page,r", [("bf16", 128, 16, 16), ("bf16", 128, 16, 1), ("bf16", 64, 32, 8), ("f32", 64, 64, 64), ("f32", 128, 24, 12)])
def test_rows_taken_back(fmt, dtype, D, page, r):
    """Rounds of up to 7 rows, some accepted: codes and scales bit for bit those of the formula after each, with
    rejected rows 2^6 larger than the others; what stays is within a step of its block's scale (int8) or 2^-4 of
    itself and e4m3's smallest step."""
    lens = [0, 3, r, 5 * r + 2]
    B = len(lens)
    import paper_2602_01762_gb300 as pkg
    h, cache, *_ = append_case(pkg, D=D, dtype=dtype, fmt=fmt, page=page, r=r, lens=lens, counts=[90] * B, Hkv=2, Hq=4)
    g = torch.Generator().manual_seed(r)
    cache.k_scales.fill_(2.0 ** -8)
    cache.v_scales.fill_(2.0 ** -8)
    rope, kept = identity_rope(400, D), [{} for _ in range(B)]
    for step in range(8):
        n = int(torch.randint(2, 8, (1,), generator=g))
        accepted = [int(torch.randint(0, n + 1, (1,), generator=g)) for _ in range(B)]
        q, k, v = (torch.randn(B, n, H, D, generator=g) for H in (4, 2, 2))
        for b, a in enumerate(accepted):
            k[b, a:] *= 64
            v[b, a:] *= 64
        q, k, v = (x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda() for x in (q, k, v))
        want = [stored(cache, name, lens, x, [n] * B, fmt) for name, x in (("k", k), ("v", v))]
        h.append(cache, q, k, v, torch.empty_like(q), rope)
        assert h.status() == 0
        for (codes, scales), name in zip(want, "kv"):
            assert torch.equal(getattr(cache, name + "_scales").cpu().double(), scales), (step, name)
            assert torch.equal(ref.codes_of(getattr(cache, name + "_pages")), codes), (step, name)
        for b, a in enumerate(accepted):
            kept[b].update({lens[b] + i: v[b, i].cpu().double() for i in range(a)})
            lens[b] += a
        cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    table, vals, scales = cache.block_table.cpu(), ref.values(cache.v_pages, cache.v_scales), cache.v_scales.cpu().double()
    for b in range(B):
        for slot, x in kept[b].items():
            p, row = int(table[b, slot // page]), slot % page
            s = scales[p, :, row // r][:, None]
            # int8: half a step of the last scale and less than half of those before together; e4m3: one rounding, and
            # steps of 2^-9 s where the scale grew past the value
            bound = s if fmt == "int8" else 2.0 ** -4 * x.abs() + 2.0 ** -9 * s
            assert ((vals[p, :, row] - x).abs() <= bound).all(), (b, slot)
    h.close()
