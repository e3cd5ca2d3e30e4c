"""Attention to a sliding window and a few first rows over a cache of the handle's own
type, against the 64-bit form (codes_ref.py)."""
from __future__ import annotations

import pytest
import torch

from . import codes_ref as ref
from .paged_ref import U, within

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def pkg():
    import paper_2602_01762_gb300 as p
    return p


def check(pkg, *, Hq, Hkv, D, dtype, page, lens, window, sinks, track=False, seed=0, hide=True):
    g = torch.Generator().manual_seed(seed)
    B, pages = len(lens), max(1, -(-max(lens) // page)) + 1
    n_pages = B * pages + 3
    table = torch.randperm(n_pages, generator=g).to(torch.int32)[:B * pages].view(B, pages).contiguous()
    k, v = (torch.randn(n_pages, Hkv, page, D, generator=g).to(DT[dtype]) for _ in range(2))
    seen = torch.zeros(n_pages, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        j = ref.seen(n, window, sinks)
        seen[table[b].long()[j // page], j % page] = True
    true_table = table.clone()
    if hide:                             # rows that are not seen are NaN, entries of pages without one lead nowhere
        k, v = (x.masked_fill(~seen[:, None, :, None], float("nan")) for x in (k, v))
        for b in range(B):
            lost = ~seen[table[b].long()].any(1)
            table[b][lost] = -5 if b % 2 else 2 ** 31 - 1
    w = torch.rand(n_pages, Hkv, page, generator=g).cuda() if track else None
    q = (torch.randn(B, Hq, D, generator=g) * 1.5).to(DT[dtype]).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((B, Hq), 7.0, device="cuda")
    h = pkg.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=B, max_pages=pages, track_weights=track)
    cache = h.cache(k.cuda(), v.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), weights=w)
    before = None if w is None else w.cpu().double()
    h.attend(cache, q, out, lse=lse, added=0, window=window, sinks=sinks)
    assert h.status() == 0
    o, l, weights, to, tl, tw = ref.attend(q, k, v, true_table, lens, D ** -0.5, window, sinks)
    within(out.cpu(), o, to, "out")
    within(lse.cpu(), l, tl, "lse")
    if track:
        want, tol = before.clone(), 4 * U * before
        for b, n in enumerate(lens):
            j = ref.seen(n, window, sinks)
            p = true_table[b].long()[j // page]
            want[p, :, j % page] += weights[b].T
            tol[p, :, j % page] += (tw[b] + 2 * U * weights[b]).T
        tol[~seen[:, None].expand_as(tol)] = 0          # unseen rows keep their weights to the bit
        within(w.cpu(), want, tol, "weights")
    first = out.clone()
    h.attend(cache, q, out, lse=lse, added=0, window=window, sinks=sinks)
    assert torch.equal(out, first)
    h.close()


LENS = [0, 1, 63, 64, 65, 128, 200, 700]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (1, 0), (1, 1), (17, 4), (64, 0), (64, 64), (65, 63), (130, 129), (128, 200), (699, 0), (700, 3), (5000, 0)])
def test_windows(pkg, dtype, window, sinks):
    check(pkg, Hq=8, Hkv=2, D=128, dtype=dtype, page=16, lens=LENS, window=window, sinks=sinks)
    check(pkg, Hq=4, Hkv=1, D=64, dtype=dtype, page=24, lens=[333], window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (8, 1), (16, 1), (20, 1), (25, 1)])
def test_groups_with_weights(pkg, dtype, D, Hq, Hkv):
    check(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=16, lens=LENS, window=70, sinks=3, track=True)


@pytest.mark.parametrize("page", [1, 5, 64, 200])
def test_pages(pkg, page):
    check(pkg, Hq=8, Hkv=2, D=64, dtype="bf16", page=page, lens=LENS, window=100, sinks=66, track=True, seed=page)


@pytest.mark.parametrize("B", [33, 129])
def test_batches(pkg, B):
    lens = [(37 * i * i + 11) % 331 for i in range(B)]
    check(pkg, Hq=8, Hkv=2, D=64, dtype="bf16", page=16, lens=lens, window=50, sinks=4, track=True)


@pytest.mark.parametrize("dtype,lens,window", [("bf16", [40007, 90], 20000), ("bf16", [100003], 1024), ("f32", [9001, 0, 5000], 4097)])
def test_long_sequences(pkg, dtype, lens, window):
    check(pkg, Hq=8, Hkv=2, D=128, dtype=dtype, page=64, lens=lens, window=window, sinks=16, hide=False)


def test_a_window_of_every_row_is_the_plain_call(pkg):
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(8, 2, 16, 64, generator=g).cuda() for _ in range(2))
    q = torch.randn(2, 4, 64, generator=g).cuda()
    h = pkg.PagedAttention(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="f32", page_size=16, max_batch=2, max_pages=4)
    cache = h.cache(k, v, torch.arange(8, dtype=torch.int32).view(2, 4).cuda(), torch.tensor([63, 10], dtype=torch.int32).cuda())
    outs = []
    for kw in (dict(), dict(window=64), dict(window=2 ** 40, sinks=2 ** 40), dict(window=30, sinks=40)):
        out = torch.zeros_like(q)
        h.attend(cache, q, out, **kw)
        outs.append(out)
    assert all(torch.equal(outs[0], x) for x in outs[1:])
    lib = h.lib
    assert lib.prism_paged_attend_window(h.h, cache.ref, 1, 5, -1, q.data_ptr(), outs[0].data_ptr(), None, None) == 1
    assert b"sinks" in lib.prism_paged_error(h.h)
    h.close()
