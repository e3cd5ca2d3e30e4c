"""What the attention over an 8-bit cache keeps of its bits: inputs whose large parts
cancel, so that a part of a probability or a query that is left out shows in the
result.  u = 2^-24, half an fp32 ulp."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def attend(Hkv, D, q, k, v, n, scale, k_scales, v_scales, table=None):
    """Output and lse of sequences of n rows each over codes k, v [pages, Hkv, page, D], one run of pages a sequence (or the given table)."""
    import paper_2602_01762_gb300 as p
    B, Hq, _ = q.shape
    page = k.shape[2]
    cols = -(-n // page)
    if table is None:
        table = torch.arange(B * cols, dtype=torch.int32, device="cuda").view(B, cols)
    h = p.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype="bf16" if q.dtype is torch.bfloat16 else "f32", page_size=page,
                         max_batch=B, max_pages=cols, softmax_scale=scale)
    cache = h.cache(k, v, table, torch.full((B,), n, dtype=torch.int32, device="cuda"), k_scales=k_scales, v_scales=v_scales)
    out, lse = torch.empty_like(q), torch.empty(B, Hq, device="cuda")
    h.attend(cache, q, out, lse=lse, added=0)
    assert h.status() == 0
    h.close()
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 12, 16, 24])
def test_probabilities_keep_their_bits(dtype, D, G):
    """Four rows of one code 64 and, by a scale for each row, values that cancel: out = sum p v / sum p is what the
    roundings of p s and of the sums leave.

    A score is one product (exact) of at most 3.  Scale, base-2 score and difference 3 u 4.4 ln 2 = 10 u of p, exp2 4 u, the
    product with the scale and its base 2 u, two parts in bf16 4 u, three accumulations and whatever they align away 16 u:
    36 u sum(p |v|) / sum p.  A bf16 result adds half its ulp.
    """
    B, Hkv, n, page, dt = 256, 2, 4, 4, DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(G)
    q = torch.zeros(B, Hkv * G, D, dtype=dt, device="cuda")
    q[..., 0] = (torch.rand(B, Hkv * G, generator=g, device="cuda") + 0.5).bfloat16().to(dt)
    k = torch.zeros(B, Hkv, page, D, dtype=torch.int8, device="cuda")
    k[..., 0] = torch.randint(-127, 0, (B, Hkv, page), generator=g, device="cuda").to(torch.int8)
    ks = torch.full((B, Hkv, page), 2.0 ** -6, device="cuda")
    z = q[..., 0].double().view(B, Hkv, G, 1) * (k[:, :, None, :, 0].double() * 2.0 ** -6)
    head = torch.randint(0, G, (B, Hkv), generator=g, device="cuda")       # the head whose values cancel
    p = torch.exp(z).gather(2, head[..., None, None].expand(B, Hkv, 1, n))[:, :, 0]
    sign = torch.tensor([1, -1, 1, -1], device="cuda", dtype=torch.float64)
    vs = torch.zeros(B, Hkv, page, device="cuda")
    vs[..., 0] = torch.rand(B, Hkv, generator=g, device="cuda") / 2 + 0.5
    vs[..., 2] = vs[..., 0] * 2.0 ** -9
    for j in (1, 3):
        vs[..., j] = (p[..., j - 1] * vs[..., j - 1].double() / p[..., j]).float()
    v = (64 * sign).to(torch.int8)[None, None, :, None].expand(B, Hkv, page, D).contiguous()
    out, _ = attend(Hkv, D, q, k, v, n, 1.0, ks, vs)
    p = torch.softmax(z, -1)
    vd = 64 * sign * vs.double()
    want = (p * vd[:, :, None]).sum(-1).view(B, Hkv * G, 1)
    tol = 36 * U * (p * vd.abs()[:, :, None]).sum(-1).view(B, Hkv * G, 1)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * want.abs()
    worst = float(((out.double() - want).abs() / tol).max())
    assert worst <= 1, worst


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
def test_long_sums_do_not_drift(D, G):
    """bf16: a scale of 2^14 enters every warp's sums at its first tile and leaves at its last, small values in between.

    All keys are 0: every p is 1.  A tile of 16 rows is added at an ulp of 2^-9 of code times scale: N / 16 roundings to
    nearest of deviation 2^-9 / sqrt(12), six of these, one whole ulp for each of the eight tiles with 2^14 in them, and half
    an ulp of the bf16 result.  Sums that drop the low bits of each tile instead lose half an ulp every time.
    """
    Hkv, n, rows = 8, 4096, 32
    B = max(1, 2 * torch.cuda.get_device_properties(0).multi_processor_count // Hkv)
    g = torch.Generator(device="cuda").manual_seed(G)
    k = torch.zeros(1, Hkv, n, D, dtype=torch.int8, device="cuda")
    v = torch.randint(64, 128, (1, Hkv, n, D), generator=g, device="cuda").to(torch.int8)
    vs = torch.full((1, Hkv, n), 2.0 ** -17, device="cuda")
    for t in range(4):
        v[:, :, t * rows], vs[:, :, t * rows] = 64, 2.0 ** 8
        v[:, :, n - (t + 1) * rows], vs[:, :, n - (t + 1) * rows] = -64, 2.0 ** 8
    q = torch.randn(B, Hkv * G, D, generator=g, device="cuda").bfloat16()
    out, _ = attend(Hkv, D, q, k, v, n, None, torch.ones(1, Hkv, n, device="cuda"), vs, torch.zeros(B, 1, dtype=torch.int32, device="cuda"))
    want = (v[0].double() * vs[0].double()[..., None]).mean(1)[None, :, None].expand(B, Hkv, G, D).reshape(B, Hkv * G, D)
    tol = (6 * (n / 16 / 12) ** 0.5 * 2.0 ** -9 + 8 * 2.0 ** -9) / n + 2.0 ** -8 * want.abs()
    worst = float(((out.double() - want).abs() / tol).max())
    assert worst <= 1, worst
    assert n / 16 * 2.0 ** -10 / n > float(tol.max())       # what a drift would add is more than is allowed


@pytest.mark.parametrize("fmt", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 8, 12, 16])
def test_fp32_queries_keep_their_bits(fmt, D, G):
    """fp32 scores of which 2^-15 and less is left when their large products cancel: a (1 + g + e) - a (1 + g + e'), a a code, e
    below 2^-15 in steps of 2^-23; lse of one row is its score.  Products up to 1.1 in size, rounded or cut at 8 places, 8 * 4.4 u."""
    B, Hkv = 64, 2
    g = torch.Generator(device="cuda").manual_seed(G)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    bits = lambda x, n: torch.round(x * 2.0 ** n) * 2.0 ** -n  # noqa: E731
    q = torch.zeros(B, Hkv, G, D, dtype=torch.float64, device="cuda")
    at = int(torch.randint(0, D // 4, (1,), generator=g, device="cuda")) * 4
    q[..., at] = 1 + bits(2.0 ** -8 * (1 + rand(B, Hkv, G) * 0.9), 15)
    q[..., at + 1] = q[..., at]
    q[..., at] += bits(2.0 ** -15 * rand(B, Hkv, G), 23)
    q[..., at + 1] += bits(2.0 ** -15 * rand(B, Hkv, G), 23)
    assert torch.equal(q.float().double(), q)
    a = torch.randint(8, 16, (B, Hkv), generator=g, device="cuda").float()      # codes of both formats
    k = torch.zeros(B, Hkv, 8, D, device="cuda")
    k[:, :, 0, at], k[:, :, 0, at + 1] = a, -a
    v = torch.ones(B, Hkv, 8, D, device="cuda")
    ks, scale = torch.full((B, Hkv, 1), 1 / 16, device="cuda"), 2.0 ** 15
    _, lse = attend(Hkv, D, q.view(B, Hkv * G, D).float(), k.to(fmt), v.to(fmt), 1, scale, ks, torch.ones_like(ks))
    want = ((q @ (k[:, :, :1].double() / 16).transpose(2, 3))[..., 0] * scale).view(B, Hkv * G)
    tol = 8 * 4.4 * U * scale + 8 * U * want.abs()
    worst = float(((lse.double() - want).abs() / tol).max())
    assert worst <= 1, worst
    assert float(want.abs().max()) > 4 * tol.max()


def test_offsets_beyond_32_bits():
    """Rows of pages past 4 GB of codes: appended, read back and attended to."""
    import paper_2602_01762_gb300 as p
    Hkv, D, page = 8, 128, 16
    n_pages = 2 ** 32 // (Hkv * page * D) + 50
    k, v = (torch.empty(n_pages, Hkv, page, D, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(n_pages, Hkv, 1, device="cuda") for _ in range(2))
    h = p.PagedAttention(n_q_heads=8, n_kv_heads=Hkv, head_dim=D, page_size=page, max_batch=2, max_pages=4)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7, 0], [n_pages - 2, n_pages - 3, 5, 6]], dtype=torch.int32, device="cuda")
    kv_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache = h.cache(k, v, table, kv_len, k_scales=ks, v_scales=vs)
    g = torch.Generator(device="cuda").manual_seed(0)
    q, x, y = (torch.randn(2, 50, 8, D, generator=g, device="cuda").bfloat16() for _ in range(3))
    rope = torch.zeros(64, 2, D // 2, device="cuda")
    rope[:, 0] = 1
    h.append(cache, q, x, y, torch.empty_like(q), rope)
    kr, vr = torch.zeros_like(x), torch.zeros_like(y)
    h.read(cache, kr, vr)
    for got, want in ((kr, x), (vr, y)):
        assert ((got.float() - want.float()).abs() <= 8 / 127 / 2 + 2.0 ** -8 * 4).all()     # values below 8: steps of at most 2^-4
    kv_len.fill_(50)
    out = torch.empty(2, 8, D, dtype=torch.bfloat16, device="cuda")
    h.attend(cache, q[:, 0].contiguous(), out, added=0)
    assert h.status() == 0
    z = torch.einsum("bhd,bnhd->bhn", q[:, 0].double(), kr.double()) * D ** -0.5
    want = torch.einsum("bhn,bnhd->bhd", torch.softmax(z, -1), vr.double())
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -8).all()   # kr and vr were rounded to bf16
    h.close()
