"""What the paged attention keeps of its bits: inputs whose large parts cancel, so
that a part of a probability, a query, a key or a value that is left out shows in
the result.  u = 2^-24, half an fp32 ulp."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def attend(Hkv, D, q, k, v, n, scale, batch_table=None):
    """Output and lse of sequences of n rows each; k, v [pages, Hkv, page, D], one run of pages a sequence (or the given table)."""
    import paper_2602_01762_gb300 as p
    B, Hq, _ = q.shape
    page = k.shape[2]
    cols = -(-n // page)
    if batch_table is None:
        batch_table = torch.arange(B * cols, dtype=torch.int32, device="cuda").view(B, cols)
    h = p.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype="bf16" if q.dtype is torch.bfloat16 else "f32", page_size=page,
                         max_batch=B, max_pages=cols, softmax_scale=scale)
    cache = h.cache(k, v, batch_table, torch.full((B,), n, dtype=torch.int32, device="cuda"))
    out, lse = torch.empty_like(q), torch.empty(B, Hq, device="cuda")
    h.attend(cache, q, out, lse=lse, added=0)
    assert h.status() == 0
    h.close()
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 12, 16, 24])
def test_probabilities_keep_their_bits(dtype, D, G):
    """Five rows whose values cancel: out = sum p v / sum p is what the roundings of p and of the sums leave.

    A score is one product (exact) of at most 3.  Scale, base-2 score and difference 3 u 4.4 ln 2 = 10 u of p, exp2 4 u, three
    accumulations and whatever they align away 16 u: 32 u sum(p |v|) / sum p.  A bf16 result adds half its ulp.
    """
    B, Hkv, n, page, dt = 256, 2, 5, 8, DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(G)
    q = torch.zeros(B, Hkv * G, D, dtype=dt, device="cuda")
    q[..., 0] = (torch.rand(B, Hkv * G, generator=g, device="cuda") + 0.5).bfloat16().to(dt)
    k = torch.zeros(B, Hkv, page, D, dtype=dt, device="cuda")
    k[..., 0] = (-2 * torch.rand(B, Hkv, page, generator=g, device="cuda")).bfloat16().to(dt)
    z = q[..., 0].double().view(B, Hkv, G, 1) * k[:, :, None, :n, 0].double()
    p = torch.exp(z)[:, :, torch.arange(D) % G]            # [B, Hkv, D, n]: dim d's values cancel for head d % G
    v = torch.zeros(B, Hkv, page, D, dtype=dt, device="cuda")
    v[:, :, 0] = (torch.rand(B, Hkv, D, generator=g, device="cuda") / 2 + 0.5).to(dt)
    left = p[..., 0] * v[:, :, 0].double()
    for j in range(1, n):
        v[:, :, j] = (-left / p[..., j]).to(dt)
        left = left + p[..., j] * v[:, :, j].double()
    out, _ = attend(Hkv, D, q, k, v, n, 1.0)
    p = torch.softmax(z, -1)
    want = (p @ v[:, :, :n].double()).view(B, Hkv * G, D)
    got = out.double()
    tol = 32 * 2.0 ** -24 * (p @ v[:, :, :n].double().abs()).view(B, Hkv * G, D)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * want.abs()
    worst = float(((got - want).abs() / tol).max())
    assert worst <= 1, worst
