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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
def test_long_sums_do_not_drift(D, G):
    """bf16: 2^14 enters every warp's sums at its first tile and leaves at its last, small values in between.

    All keys are 0: every p is 1.  A tile of r rows is added at an ulp of 2^-9: N / r roundings to nearest of deviation
    2^-9 / sqrt(12), six of these (1e-9 of all results beyond), one whole ulp for each of the eight tiles with 2^14 in
    them, and half an ulp of the bf16 result.  Sums that drop the low bits of each tile instead lose half an ulp every time,
    N / r 2^-10.
    """
    ctas = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    Hkv, n = 8, 4096
    B = max(1, ctas // Hkv)                                # about a segment to every CTA
    rows = 16 if D == 128 else 32
    g = torch.Generator(device="cuda").manual_seed(G)
    k = torch.zeros(1, Hkv, n, D, dtype=torch.bfloat16, device="cuda")
    v = ((torch.rand(1, Hkv, n, D, generator=g, device="cuda") + 1) * 2.0 ** -11).bfloat16()
    for t in range(4):
        v[:, :, t * rows] = 2.0 ** 14
        v[:, :, n - (t + 1) * rows] = -2.0 ** 14
    q = torch.randn(B, Hkv * G, D, generator=g, device="cuda").bfloat16()
    out, _ = attend(Hkv, D, q, k, v, n, None, batch_table=torch.zeros(B, 1, dtype=torch.int32, device="cuda"))
    want = v[0].double().mean(1)[None, :, None].expand(B, Hkv, G, D).reshape(B, Hkv * G, D)
    tol = (6 * (n / rows / 12) ** 0.5 * 2.0 ** -9 + 8 * 2.0 ** -9) / n + 2.0 ** -8 * want.abs()
    worst = float(((out.double() - want).abs() / tol).max())
    assert worst <= 1, worst
    assert n / rows * 2.0 ** -10 / n > float(tol.max())     # what a drift would add is more than is allowed


U = 2.0 ** -24


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 8, 12, 16])
@pytest.mark.parametrize("what", ["keys", "queries", "both"])
def test_fp32_scores_keep_their_bits(what, D, G):
    """fp32 scores of which 2^-15 and less is left when their large products cancel; lse of one row is that row's score.

    keys: a (1 + g + e) - a (1 + g + e'), queries the same with the sides exchanged, e below 2^-15 in steps of 2^-23; both: (a + f) (c + g)
    - (a + f) c - a (c + g) + a c = f g.  Products up to 1.1 in size, four at most: rounded or cut at 8 places, 8 * 4.4 u.
    """
    B, Hkv = 64, 2
    g = torch.Generator(device="cuda").manual_seed(G)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    bits = lambda x, n: torch.round(x * 2.0 ** n) * 2.0 ** -n  # noqa: E731
    q = torch.zeros(B, Hkv, G, D, dtype=torch.float64, device="cuda")
    k = torch.zeros(B, Hkv, 1, D, dtype=torch.float64, device="cuda")
    at = int(torch.randint(0, D // 4, (1,), generator=g, device="cuda")) * 4
    if what == "both":
        f, s = bits(2.0 ** -9 * (1 + rand(B, Hkv, G) * 0.9), 16), bits(2.0 ** -8 * (1 + rand(B, Hkv, 1) * 0.9), 15)
        for d, (x, y) in enumerate(((1 + f, 1 + s), (1 + f, -torch.ones_like(s)), (torch.ones_like(f), -1 - s), (torch.ones_like(f), torch.ones_like(s)))):
            q[..., at + d], k[..., at + d] = x, y
    else:
        a, b = (q, k) if what == "keys" else (k, q)
        a[..., at] = bits(0.9 + 0.2 * rand(*a.shape[:3]), 20)
        a[..., at + 1] = -a[..., at]
        b[..., at] = 1 + bits(2.0 ** -8 * (1 + rand(*b.shape[:3]) * 0.9), 15)
        b[..., at + 1] = b[..., at]
        b[..., at] += bits(2.0 ** -15 * rand(*b.shape[:3]), 23)
        b[..., at + 1] += bits(2.0 ** -15 * rand(*b.shape[:3]), 23)
    assert torch.equal(q.float().double(), q) and torch.equal(k.float().double(), k)
    scale = 2.0 ** 15
    v = torch.ones(B, Hkv, 8, D, device="cuda")
    page = torch.zeros(B, Hkv, 8, D, device="cuda")
    page[:, :, :1] = k.float()
    _, lse = attend(Hkv, D, q.view(B, Hkv * G, D).float(), page, v, 1, scale)
    want = ((q @ k.transpose(2, 3))[..., 0] * scale).view(B, Hkv * G)
    tol = 8 * 4.4 * U * scale + 8 * U * want.abs()
    worst = float(((lse.double() - want).abs() / tol).max())
    assert worst <= 1, worst
    assert float(want.abs().max()) > 4 * tol.max()          # what the parts below hold is well above the bound


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 8, 12, 16])
def test_fp32_values_keep_their_bits(D, G):
    """Two rows of equal scores whose values differ in their last bits alone: half that difference, to 8 u."""
    B, Hkv, page = 16, 2, 8
    g = torch.Generator(device="cuda").manual_seed(G)
    k = torch.zeros(B, Hkv, page, D, device="cuda")
    v = torch.zeros(B, Hkv, page, D, device="cuda")
    v[:, :, :2] = 1 + torch.round(torch.rand(B, Hkv, 1, D, generator=g, device="cuda") * 2 ** 7) * 2.0 ** -15
    v[:, :, :2] += torch.round(torch.rand(B, Hkv, 2, D, generator=g, device="cuda") * 2 ** 8) * 2.0 ** -23
    v[:, :, 1].neg_()
    q = torch.randn(B, Hkv * G, D, generator=g, device="cuda")
    out, _ = attend(Hkv, D, q, k, v, 2, None)
    want = (v[:, :, :2].double().sum(2) / 2)[:, :, None].expand(B, Hkv, G, D).reshape(B, Hkv * G, D)
    assert float((out.double() - want).abs().max()) <= 8 * U
    assert float(want.abs().max()) > 64 * U
