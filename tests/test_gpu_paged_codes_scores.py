"""Attention over codes where scores are so large that log2 of a scale is lost beside
them: each row's weight goes by its own scale all the same."""
from __future__ import annotations

import pytest
import torch

from . import codes_ref as ref
from .test_gpu_paged_codes import DT

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 24, 2.0 ** 26, 2.0 ** 34, 2.0 ** 60])
@pytest.mark.parametrize("low,high", [(6, 6), (12, 12), (-40, 12), (-60, -60), (0, 100)])
def test_equal_scores_of_any_size(low, high, size, sign):
    """Rows of one key: every score is the same and every p one number, so that out is the mean of the values.

    The sum of p has some 12 additions in a lane, 3 between lanes, 4 of warps and up to 8 of CTAs, the sums of p v as many,
    inverse and product two more: 64 u of sum |v| / n, beside the weights' 2^-22 (bf16, two parts) or 2^-24 and what fp16
    leaves below a tile's largest weight, 2^-36 of it for each code; lse: the score's three roundings and two more."""
    n, page, D = 333, 16, 64
    for dtype in DT:
        for Hq, fmt in ((4, "e4m3"), (8, "int8"), (16, "e4m3"), (6, "int8")):
            g = torch.Generator().manual_seed(Hq)
            import paper_2602_01762_gb300 as p
            cols = -(-n // page)
            k = torch.full((cols, 1, page, D), 64.0)
            v = torch.randint(-12, 13, (cols, 1, page, D), generator=g).float()
            v = v.to(ref.TYPE[fmt])
            ks = torch.ones(cols, 1, 2)
            vs = torch.exp2(torch.randint(low, high + 1, (cols, 1, 2), generator=g).float())
            q = torch.full((1, Hq, D), 4.0 * sign, dtype=DT[dtype], device="cuda")
            h = p.PagedAttention(n_q_heads=Hq, n_kv_heads=1, head_dim=D, dtype=dtype, page_size=page, max_batch=1, max_pages=cols,
                                 softmax_scale=size / (64 * 4 * 64))
            cache = h.cache(k.to(ref.TYPE[fmt]).cuda(), v.cuda(), torch.arange(cols, dtype=torch.int32, device="cuda")[None],
                            torch.tensor([n], dtype=torch.int32, device="cuda"), k_scales=ks.cuda(), v_scales=vs.cuda())
            out, lse = torch.empty_like(q), torch.empty(1, Hq, device="cuda")
            h.attend(cache, q, out, lse=lse, added=0)
            assert h.status() == 0
            h.close()
            x = ref.values(v, vs)[:, 0].reshape(-1, D)[:n]
            codes = ref.codes_of(v)[:, 0].reshape(-1, D)[:n]
            want = x.mean(0)
            tol = (64 * U + 2.0 ** -22) * x.abs().mean(0) + 2.0 ** -36 * float(vs.max()) * codes.abs().mean(0)
            tol = tol + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
            worst = float(((out[0].cpu().double() - want).abs() / tol).max())
            assert worst <= 1, (dtype, Hq, fmt, worst)
            exact = sign * size + torch.log(torch.tensor(float(n), dtype=torch.float64))
            assert float((lse.cpu().double() - exact).abs().max()) <= 6 * U * size + 2.0 ** -18, (dtype, Hq)


@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 25, 2.0 ** 33])
def test_scores_that_grow_by_more_than_they_hold(size):
    """Keys ever larger: the last one's row alone counts, whatever the scales of those before."""
    n, page, D = 70, 1, 64
    import paper_2602_01762_gb300 as p
    for dtype in DT:
        for Hq in (4, 8, 16):
            for order in (1, -1):
                k = torch.arange(1, n + 1).sort(descending=order < 0)[0].view(n, 1, 1, 1).expand(n, 1, 1, D).contiguous().to(torch.int8)
                v = torch.arange(n).view(n, 1, 1, 1).expand(n, 1, 1, D).contiguous().to(torch.int8)
                vs = torch.exp2((torch.arange(n) * 29 % 41 - 20).float()).view(n, 1, 1)
                q = torch.full((1, Hq, D), 1.0, dtype=DT[dtype], device="cuda")
                h = p.PagedAttention(n_q_heads=Hq, n_kv_heads=1, head_dim=D, dtype=dtype, page_size=page, max_batch=1, max_pages=n, softmax_scale=size / D)
                cache = h.cache(k.cuda(), v.cuda(), torch.arange(n, dtype=torch.int32, device="cuda")[None],
                                torch.tensor([n], dtype=torch.int32, device="cuda"), k_scales=torch.ones(n, 1, 1, device="cuda"), v_scales=vs.cuda())
                out = torch.empty_like(q)
                h.attend(cache, q, out, added=0)
                h.close()
                top = n - 1 if order == 1 else 0
                want = float(vs[top]) * top
                # scores differ by `size` at least: exp(-2^10) is 0
                assert float((out.double() - want).abs().max()) <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) * want, (dtype, Hq, order)


@pytest.mark.parametrize("rows", ["one", "some", "all"])
def test_infinite_scores(rows):
    """A score of -inf drops its row (all of them: zeros and -inf), one of +inf makes its head NaN and no other."""
    import paper_2602_01762_gb300 as p
    n, page, D, Hkv = 200, 16, 64, 2
    cols = -(-n // page)
    for dtype in DT:
        for G, fmt in ((4, "int8"), (8, "e4m3"), (12, "int8")):
            g = torch.Generator().manual_seed(G)
            k = torch.randint(1, 13, (cols, Hkv, page, D), generator=g).float()
            v = torch.randint(-12, 13, (cols, Hkv, page, D), generator=g).float()
            ks, vs = (torch.exp2(torch.randint(-6, -3, (cols, Hkv, page), generator=g).float()) for _ in range(2))
            slots = {"one": [37], "some": [0, 16, 17, 40, 99, 199], "all": list(range(n))}[rows]
            at = [(s // page, s % page) for s in slots]
            for c, r in at:
                ks[c, 0, r] = float("inf")
            q = torch.rand(2, Hkv * G, D, generator=g) + 0.5
            q[0, :G] *= -1                                       # -inf where ks is infinite; the second sequence +inf
            q = q.to(DT[dtype]).cuda()
            h = p.PagedAttention(n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=2, max_pages=cols)
            table = torch.arange(cols, dtype=torch.int32, device="cuda")[None].expand(2, -1).contiguous()
            cache = h.cache(k.to(ref.TYPE[fmt]).cuda(), v.to(ref.TYPE[fmt]).cuda(), table, torch.full((2,), n, dtype=torch.int32, device="cuda"),
                            k_scales=ks.cuda(), v_scales=vs.cuda())
            out, lse = torch.empty_like(q), torch.empty(2, Hkv * G, device="cuda")
            h.attend(cache, q, out, lse=lse, added=0)
            assert h.status() == 0
            h.close()
            assert torch.isnan(out[1, :G]).all() and torch.isnan(lse[1, :G]).all()
            x, y = (t.permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n] for t in (ref.values(k, ks), ref.values(v, vs)))
            for b in range(2):
                for head in range(Hkv):
                    if b == 1 and head == 0:
                        continue
                    z = q[b, head * G:(head + 1) * G].cpu().double() @ x[head].T * D ** -0.5
                    got, got_lse = out[b, head * G:(head + 1) * G].cpu().double(), lse[b, head * G:(head + 1) * G].cpu().double()
                    if torch.isinf(z).all():
                        assert (got == 0).all() and (got_lse == -float("inf")).all()
                        continue
                    w = torch.softmax(z, -1)
                    # scores of at most 2^9, whose fp32 sums and scaling err by 2^-12 at most
                    tol = 2.0 ** -10 * (w @ y[head].abs()) + (2.0 ** -8 * (w @ y[head]).abs() if dtype == "bf16" else 0.0)
                    assert ((got - w @ y[head]).abs() <= tol).all() and ((got_lse - torch.logsumexp(z, -1)).abs() <= 2.0 ** -10).all()
