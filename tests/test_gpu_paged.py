"""The paged-cache operators on the GPU against their 64-bit forms (paged_ref.py)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from . import paged_ref as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def pkg():
    import paper_2602_01762_gb300 as p
    return p


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


def pool(g, n_pages, Hkv, page, D, dtype, layout):
    """K and V pages in one of the storage orders a program may have."""
    if layout == "heads_first":
        return normal(g, n_pages, Hkv, page, D, dtype=dtype), normal(g, n_pages, Hkv, page, D, dtype=dtype)
    if layout == "rows_first":       # [page, row, head, D]
        return tuple(normal(g, n_pages, page, Hkv, D, dtype=dtype).transpose(1, 2) for _ in range(2))
    both = normal(g, n_pages, 2, Hkv, page, D, dtype=dtype)   # K and V of a page side by side
    return both[:, 0], both[:, 1]


def tables(g, B, pages, spare=3):
    """A shuffled block table over a pool with pages that belong to nobody."""
    n = B * pages + spare
    return n, torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:B * pages].view(B, pages).contiguous()


def poison_unused(pages, table, lens, page):
    """NaN into every row that no sequence holds."""
    keep = torch.zeros(pages.shape[0], page, dtype=torch.bool)
    for b, n in enumerate(lens):
        for j in range(n):
            keep[int(table[b, j // page]), j % page] = True
    pages.masked_fill_(~keep.cuda()[:, None, :, None], float("nan"))


def attend_case(pkg, *, Hq, Hkv, D, dtype, page, lens, layout="heads_first", track=False, scale=None, seed=0, qscale=1.5,
                wild=True):
    g = rng(seed)
    B, dt = len(lens), DT[dtype]
    pages = max(1, -(-max(lens) // page)) + 1
    n_pages, table = tables(g, B, pages)
    k, v = pool(g, n_pages, Hkv, page, D, dt, layout)
    if wild:
        for t in (k, v):
            poison_unused(t, table.cpu(), lens, page)
        for b, n in enumerate(lens):           # entries past a sequence's rows are never followed
            table[b, -(-n // page):] = -7 if b % 2 else 2 ** 31 - 1
    q = normal(g, B, Hq, D, dtype=dt, scale=qscale)
    out, lse = torch.full_like(q, 7.0), torch.full((B, Hq), 7.0, device="cuda")
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    w = torch.rand(n_pages, Hkv, page, generator=g, device="cuda") if track else None
    h = pkg.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=B, max_pages=pages,
                           track_weights=track, softmax_scale=scale, rms_eps=EPS)
    cache = h.cache(k, v, table, kv_len, weights=w)
    return h, cache, q, out, lse, scale if scale is not None else D ** -0.5


def check_attend(pkg, **kw):
    lens = kw["lens"]
    h, cache, q, out, lse, scale = attend_case(pkg, **kw)
    before = None if cache.weights is None else cache.weights.clone()
    h.attend(cache, q, out, lse=lse, added=0)
    assert h.status() == 0
    o, l, w, to, tl, tw = ref.attend(q, cache.k_pages, cache.v_pages, cache.block_table, lens, scale)
    ref.within(out, o, to, "out")
    ref.within(lse, l, tl, "lse")
    if before is not None:
        want, tol = before.double(), ref.U * 4 * before.double()
        page = kw["page"]
        for b, n in enumerate(lens):
            for j0 in range(0, n, page):
                p, m = int(cache.block_table[b, j0 // page]), min(page, n - j0)
                want[p, :, :m] += w[b][:, j0:j0 + m]
                tol[p, :, :m] += tw[b][:, j0:j0 + m] + 2 * ref.U * w[b][:, j0:j0 + m]
        ref.within(cache.weights, want, tol, "weights")
    first = out.clone()
    h.attend(cache, q, out, lse=lse, added=0)
    assert torch.equal(out, first)           # the same bits again
    h.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (6, 2), (8, 2), (5, 1), (14, 2), (8, 1), (9, 1), (16, 1), (20, 1), (64, 2)])
def test_attend_groups(pkg, dtype, D, Hq, Hkv):
    check_attend(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=16, lens=[37, 300, 1], track=Hq in (6, 14, 20, 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 5, 16, 24, 64, 200])
@pytest.mark.parametrize("layout", ["heads_first", "rows_first", "interleaved"])
def test_attend_pages_and_layouts(pkg, dtype, page, layout):
    check_attend(pkg, Hq=8, Hkv=2, D=128, dtype=dtype, page=page, lens=[0, 1, 15, 16, 17, 127, 128, 129, 395], layout=layout,
                 track=True, seed=page)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 7, 8, 31, 32, 33, 63, 64, 65, 257])
def test_attend_lengths_around_tiles(pkg, D, n):
    for dtype in DT:
        check_attend(pkg, Hq=4, Hkv=1, D=D, dtype=dtype, page=8, lens=[n], track=True)


@pytest.mark.parametrize("B", [32, 33, 45, 129, 300])
def test_attend_batches(pkg, B):
    """Work is found in one warp up to 32 sequences, by the whole CTA above."""
    lens = [(37 * i * i + 11) % 331 for i in range(B)]
    check_attend(pkg, Hq=8, Hkv=2, D=64, dtype="bf16", page=16, lens=lens, track=True)
    check_attend(pkg, Hq=2, Hkv=2, D=64, dtype="f32", page=16, lens=lens, wild=False)


@pytest.mark.parametrize("dtype,lens", [("bf16", [40007]), ("bf16", [9, 20011, 0, 4999]), ("f32", [9001])])
def test_attend_long_rows_are_joined(pkg, dtype, lens):
    check_attend(pkg, Hq=8, Hkv=2, D=128, dtype=dtype, page=64, lens=lens, track=True, wild=False)


def test_attend_peaked_and_flat_scores(pkg):
    for qs in (0.0, 1e-3, 30.0):
        check_attend(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", page=16, lens=[700, 90], qscale=qs)
        check_attend(pkg, Hq=8, Hkv=2, D=128, dtype="f32", page=16, lens=[700, 90], qscale=qs)
    check_attend(pkg, Hq=8, Hkv=2, D=64, dtype="f32", page=16, lens=[77], scale=0.31)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_infinite_and_nan_values(pkg, dtype):
    """-inf scores drop a row; all of them -inf give zeros; a NaN or +inf score makes its head NaN and no other."""
    h, cache, q, out, lse, _ = attend_case(pkg, Hq=4, Hkv=2, D=64, dtype=dtype, page=16, lens=[50, 50], wild=False)
    lowest = torch.finfo(DT[dtype]).min
    q.fill_(0)
    q[..., 0] = 1.0
    q[:, 1, 0] = 0.0                       # heads 0 and 1 share KV head 0
    k, t = cache.k_pages, cache.block_table
    at = lambda b, h, j: k[int(t[b, j // 16]), h, j % 16]  # noqa: E731
    v_at = lambda b, h, j: cache.v_pages[int(t[b, j // 16]), h, j % 16]  # noqa: E731
    for j in range(50):
        at(0, 0, j)[0] = -math.inf if j != 33 else 0.5     # head 0 of sequence 0: row 33 alone counts
        at(0, 1, j)[0] = -math.inf                          # KV head 1: nothing counts
        at(1, 0, j)[0] = lowest                             # the type's lowest value everywhere: a plain average
        at(1, 1, j)[0] = math.nan if j == 20 else 1.0
    h.attend(cache, q, out, lse=lse, added=0)
    assert h.status() == 0
    assert torch.equal(out[0, 0], v_at(0, 0, 33))
    assert torch.isnan(out[0, 1]).all()                     # 0 * -inf scores
    assert (out[0, 2:] == 0).all() and (lse[0, 2:] == -math.inf).all()
    mean = torch.stack([v_at(1, 0, j).double() for j in range(50)]).mean(0)
    ref.within(out[1, 0], mean, 2.0 ** -8 * mean.abs() + 2.0 ** -15, "average")
    assert torch.isnan(out[1, 2:]).all() and torch.isfinite(out[1, :2]).all()
    h.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(9, 1), (16, 1), (13, 1), (40, 2)])
def test_attend_fp32_many_heads_over_many_rows(pkg, D, Hq, Hkv):
    """16 heads of fp32 to a pass, in shares of the grid, with and without weights."""
    check_attend(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype="f32", page=24, lens=[17, 0, 9001, 1, 8191, 33], track=Hq != 13, seed=Hq)


@pytest.mark.parametrize("D,Hq", [(64, 16), (128, 16), (64, 7), (128, 10)])
def test_attend_fp32_many_heads_short_rows(pkg, D, Hq):
    """The same in clusters: many short sequences."""
    check_attend(pkg, Hq=Hq, Hkv=1, D=D, dtype="f32", page=16, lens=[480] + [(37 * i) % 481 for i in range(69)], track=True)


@pytest.mark.parametrize("G", [8, 16])
@pytest.mark.parametrize("qscale", [0.0, 1e-3, 30.0, 1e-30])
def test_attend_fp32_parts(pkg, G, qscale):
    """Flat, peaked and vanishing scores of values in three parts."""
    check_attend(pkg, Hq=G, Hkv=1, D=128, dtype="f32", page=64, lens=[33001, 77], qscale=qscale, wild=False)
    check_attend(pkg, Hq=2 * G, Hkv=2, D=64, dtype="f32", page=8, lens=[300, 77], qscale=qscale, scale=0.31)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [5, 8, 12, 16])
@pytest.mark.parametrize("rows", [50, 33000])
def test_attend_fp32_many_heads_infinite_and_nan_values(pkg, D, G, rows):
    """Infinities have no finite parts; scores are what their definition says all the same."""
    h, cache, q, out, lse, _ = attend_case(pkg, Hq=2 * G, Hkv=2, D=D, dtype="f32", page=16, lens=[50, 50, rows], wild=False)
    lowest = torch.finfo(torch.float32).min
    k, t = cache.k_pages, cache.block_table
    q.fill_(0)
    q[..., 0] = 1.0
    q[:, 1, 0] = 0.0                       # head 1: 0 times infinity
    q[:, 2, 1] = -1.0                      # head 2: minus the second dim as well
    for j in range(50):
        at = lambda b, hd: k[int(t[b, j // 16]), hd, j % 16]  # noqa: B023,E731
        at(0, 0)[0] = -math.inf if j != 33 else 0.5
        at(0, 0)[1] = 0.25
        at(0, 1)[0] = -math.inf
        at(0, 1)[1] = 0.0
        at(1, 0)[0] = lowest
        at(1, 0)[1] = 0.0
        at(1, 1)[0] = math.nan if j == 20 else 1.0
    h.attend(cache, q, out, lse=lse, added=0)
    assert h.status() == 0
    v_at = lambda b, hd, j: cache.v_pages[int(t[b, j // 16]), hd, j % 16]  # noqa: E731
    for head in range(G):
        if head == 1:
            assert torch.isnan(out[0, head]).all() and torch.isnan(lse[0, head])
        else:
            assert torch.equal(out[0, head], v_at(0, 0, 33))
    assert (out[0, G:] == 0).all() and (lse[0, G:] == -math.inf).all()
    mean = torch.stack([v_at(1, 0, j).double() for j in range(50)]).mean(0)
    spread = torch.stack([v_at(1, 0, j).double().abs() for j in range(50)]).mean(0)
    ref.within(out[1, :G], mean.expand(G, D), 2.0 ** -19 * spread.expand(G, D), "average")
    assert torch.isnan(out[1, G:]).all() and torch.isfinite(out[1, :G]).all()
    o, l, _, to, tl, _ = ref.attend(q[2:], k, cache.v_pages, t[2:], [rows], D ** -0.5)
    ref.within(out[2:], o, to)
    ref.within(lse[2:], l, tl)
    h.close()


def test_attend_added_rows_and_other_stream(pkg):
    h, cache, q, out, lse, scale = attend_case(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", page=16, lens=[40, 129], wild=False)
    cache.kv_len.sub_(1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    h.attend(cache, q, out, lse=lse, stream=s)              # added = 1
    torch.cuda.current_stream().wait_stream(s)
    o, l, _, to, tl, _ = ref.attend(q, cache.k_pages, cache.v_pages, cache.block_table, [40, 129], scale)
    ref.within(out, o, to)
    with torch.cuda.stream(s):
        out.zero_()
        h.attend(cache, q, out, lse=None)
    s.synchronize()
    ref.within(out, o, to)
    h.close()


@pytest.mark.parametrize("what", ["page", "long", "negative"])
def test_attend_device_flags(pkg, what):
    h, cache, q, out, lse, _ = attend_case(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", page=16, lens=[40, 60], wild=False, track=True)
    if what == "page":
        cache.block_table[1, 1] = cache.k_pages.shape[0]
        bit = 16
    else:
        cache.kv_len[1] = cache.rows + 1 if what == "long" else -3
        bit = 2
    h.attend(cache, q, out, lse=lse, added=0)
    assert h.status() & bit
    assert h.status() == 0                                  # cleared
    o, _, _, to, _, _ = ref.attend(q[:1], cache.k_pages, cache.v_pages, cache.block_table[:1], [40], 128 ** -0.5)
    ref.within(out[:1], o, to)                              # the other sequence is untouched
    if what == "negative":
        assert (out[1] == 0).all()
    h.close()


def test_offsets_beyond_32_bits(pkg):
    """Rows at byte offsets above 2^32 of a pool (K and V interleaved in one)."""
    g = rng(5)
    n_pages, Hkv, page, D = 150000, 2, 64, 128              # 9.8 GB
    both = torch.empty(n_pages, 2, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    k, v = both[:, 0], both[:, 1]
    ids = [n_pages - 1, 3, n_pages // 2 + 1, n_pages - 2]
    for i in ids:
        both[i] = normal(g, 2, Hkv, page, D, dtype=torch.bfloat16)
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([200], dtype=torch.int32, device="cuda")
    h = pkg.PagedAttention(n_q_heads=8, n_kv_heads=2, head_dim=D, page_size=page, max_batch=1, max_pages=4)
    w = torch.rand(n_pages, Hkv, page, generator=g, device="cuda")
    cache = h.cache(k, v, table, kv_len)
    rope = pkg.rope_table(300, D)
    q = normal(g, 1, 1, 8, D, dtype=torch.bfloat16)
    kn, vn = normal(g, 1, 1, 2, D, dtype=torch.bfloat16), normal(g, 1, 1, 2, D, dtype=torch.bfloat16)
    qo, out = torch.empty_like(q), torch.empty(1, 8, D, dtype=torch.bfloat16, device="cuda")
    h.append(cache, q, kn, vn, qo, rope)
    y, tol = ref.norm_rope(kn[0], None, rope, 200, EPS)
    ref.within(k[n_pages - 2, :, 200 - 192], y[0], tol[0] + 2.0 ** -8 * y[0].abs())
    assert torch.equal(v[n_pages - 2, :, 200 - 192], vn[0, 0])
    h.attend(cache, qo.view(1, 8, D), out)
    o, _, _, to, _, _ = ref.attend(qo.view(1, 8, D), k, v, table, [201], D ** -0.5)
    ref.within(out, o, to)
    tracked = h.cache(k, v, table, kv_len, weights=w)
    dst = h.cache(k, v, torch.tensor([[n_pages - 5, n_pages - 6]], dtype=torch.int32, device="cuda"), torch.zeros_like(kv_len), weights=w)
    kept = torch.empty(1, 2, 100, dtype=torch.int32, device="cuda")
    h.evict(tracked, dst, kept, sinks=2, recent=10)
    assert h.status() == 0
    for hd in range(2):
        wl = ref.gather(w, table[0].cpu(), 200)[hd].cpu().numpy()
        rows = ref.kept_rows(wl, 200, 100, 2, 10)
        assert np.array_equal(kept[0, hd].cpu().numpy(), rows)
        got = ref.gather(k, dst.block_table[0], 100)[hd]
        assert torch.equal(got, ref.gather(k, table[0], 200)[hd][torch.from_numpy(rows).cuda()])
    h.close()


# ------------------------------------------------------------- norm and rotation

def rows_case(pkg, *, Hq, Hkv, D, dtype, B, n, gains, seed=0, order="fused"):
    g, dt = rng(seed), DT[dtype]
    if order == "fused":
        x = normal(g, B, n, (Hq + 2 * Hkv) * D, dtype=dt, scale=1.7)
        q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([Hq * D, Hkv * D, Hkv * D], -1))
    else:                              # [B, heads, n, D] storage
        q, k, v = (normal(g, B, h, n, D, dtype=dt, scale=1.7).transpose(1, 2) for h in (Hq, Hkv, Hkv))
    g_q, g_k = (normal(g, D, dtype=dt, scale=0.2) + 1 for _ in range(2)) if gains else (None, None)
    pos = torch.randint(0, 50, (B,), generator=g, device="cuda", dtype=torch.int32)
    n_new = torch.randint(0, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n_new[0] = n
    return q, k, v, g_q, g_k, pos, n_new, pkg.rope_table(n + 60, D, 500000.0)


def handle(pkg, Hq, Hkv, D, dtype, **kw):
    return pkg.PagedAttention(**{**dict(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=16, max_batch=1,
                                        max_pages=1, rms_eps=EPS), **kw})


def bf16_more(dtype, y):
    return 2.0 ** -8 * y.abs() if dtype == "bf16" else 0.0


SHAPES = [(4, 4, 64), (3, 1, 64), (8, 2, 128), (32, 8, 128), (7, 7, 128), (1, 1, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("gains", [True, False])
@pytest.mark.parametrize("B,n,order", [(1, 1, "fused"), (3, 5, "heads"), (2, 70, "fused"), (37, 1, "fused")])
def test_norm_rope_and_gradient(pkg, dtype, Hq, Hkv, D, gains, B, n, order):
    q, k, _, g_q, g_k, pos, n_new, rope = rows_case(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, B=B, n=n, gains=gains, order=order)
    h = handle(pkg, Hq, Hkv, D, dtype)
    g = rng(9)
    qo = torch.full((B, Hq, n, D), 7.0, dtype=DT[dtype], device="cuda").transpose(1, 2)
    ko = torch.full((B, n, Hkv, D), 7.0, dtype=DT[dtype], device="cuda")
    h.qk_norm_rope(q, k, qo, ko, rope, pos, g_q=g_q, g_k=g_k, n_new=n_new)
    dqo, dko = normal(g, B, n, Hq, D, dtype=DT[dtype], scale=0.1), normal(g, B, Hkv, n, D, dtype=DT[dtype], scale=0.1).transpose(1, 2)
    dq, dk = torch.full_like(dqo, 7.0), torch.full((B, n, Hkv, D), 7.0, dtype=DT[dtype], device="cuda")
    dg = [torch.full((D,), 7.0, device="cuda") if gains else None for _ in range(2)]
    h.qk_norm_rope_backward(dqo, dko, q, k, dq, dk, rope, pos, g_q=g_q, g_k=g_k, dg_q=dg[0], dg_k=dg[1], n_new=n_new)
    assert h.status() == 0
    for x, gain, y, dy, dx, dgain in ((q, g_q, qo, dqo, dq, dg[0]), (k, g_k, ko, dko, dk, dg[1])):
        total, tol_total = (torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(2))
        for b in range(B):
            m, p = int(n_new[b]), int(pos[b])
            want, tol = ref.norm_rope(x[b, :m], gain, rope, p, EPS)
            ref.within(y[b, :m], want, tol + bf16_more(dtype, want), "y")
            assert (y[b, m:] == 7.0).all()                  # rows past n_new are left alone
            want, dgw, tol, dgt = ref.norm_rope_grad(x[b, :m], gain, dy[b, :m], rope, p, EPS)
            ref.within(dx[b, :m], want, tol + bf16_more(dtype, want), "dx")
            assert (dx[b, m:] == 0).all()
            if gains:
                total += dgw
                tol_total += dgt
        if gains:
            ref.within(dgain, total, tol_total, "dg")
    h.close()


def test_gradient_against_differences(pkg):
    """The change of sum(dy . y) along random directions, by central differences of
    the 64-bit forward, against the kernel's gradients."""
    B, n, Hq, Hkv, D = 2, 9, 6, 2, 64
    q, k, _, g_q, g_k, pos, _, rope = rows_case(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype="f32", B=B, n=n, gains=True)
    h = handle(pkg, Hq, Hkv, D, "f32")
    g = rng(3)
    dqo, dko = normal(g, B, n, Hq, D, dtype=torch.float32), normal(g, B, n, Hkv, D, dtype=torch.float32)
    dq, dk, dg_q, dg_k = torch.empty_like(dqo), torch.empty_like(dko), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    h.qk_norm_rope_backward(dqo, dko, q, k, dq, dk, rope, pos, g_q=g_q, g_k=g_k, dg_q=dg_q, dg_k=dg_k)

    def total(x, gain, dy):
        return sum(float((ref.norm_rope(x[b], gain, rope, int(pos[b]), EPS)[0] * dy[b].double()).sum()) for b in range(B))

    step = 1e-4                                              # error step^2 times a third derivative, about 1e-8 of the change
    for x, gain, dy, dx, dgain in ((q, g_q, dqo, dq, dg_q), (k, g_k, dko, dk, dg_k)):
        for i in range(4):
            u, w = torch.randn(x.shape, generator=g, device="cuda").double(), torch.randn(D, generator=g, device="cuda").double()
            x64, g64 = x.double(), gain.double()
            for want, got, size in (
                    ((total(x64 + step * u, g64, dy) - total(x64 - step * u, g64, dy)) / (2 * step), float((dx.double() * u).sum()),
                     float((dx.double() * u).abs().sum())),
                    ((total(x64, g64 + step * w, dy) - total(x64, g64 - step * w, dy)) / (2 * step), float((dgain.double() * w).sum()),
                     float((dgain.double() * w).abs().sum()))):
                assert abs(got - want) <= 2e-6 * size + 1e-6, (got, want, size)
    h.close()


def test_gradient_many_rows_same_bits(pkg):
    """Enough rows that every SM takes part: gains' gradients against the formula, and the same bits twice."""
    B, n, Hq, Hkv, D = 3, 1500, 8, 2, 128
    q, k, _, g_q, g_k, pos, n_new, rope = rows_case(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype="bf16", B=B, n=n, gains=True)
    h = handle(pkg, Hq, Hkv, D, "bf16")
    g = rng(3)
    dqo, dko = normal(g, B, n, Hq, D, dtype=torch.bfloat16), normal(g, B, n, Hkv, D, dtype=torch.bfloat16)
    got = []
    for _ in range(3):
        dq, dk, dg = torch.empty_like(dqo), torch.empty_like(dko), torch.empty(2, D, device="cuda")
        h.qk_norm_rope_backward(dqo, dko, q, k, dq, dk, rope, pos, g_q=g_q, g_k=g_k, dg_q=dg[0], dg_k=dg[1], n_new=n_new)
        got.append((dq, dk, dg))
    for a in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(a, got[0]))
    for i, (x, gain, dy) in enumerate(((q, g_q, dqo), (k, g_k, dko))):
        parts = [ref.norm_rope_grad(x[b, :int(n_new[b])], gain, dy[b, :int(n_new[b])], rope, int(pos[b]), EPS) for b in range(B)]
        ref.within(got[0][2][i], sum(p[1] for p in parts), sum(p[3] for p in parts), "dg")
    h.close()


def test_norm_rope_in_place(pkg):
    q, k, _, g_q, g_k, pos, n_new, rope = rows_case(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", B=2, n=33, gains=True)
    h = handle(pkg, 8, 2, 128, "bf16")
    qo, ko = q.clone(), k.clone()
    h.qk_norm_rope(q, k, qo, ko, rope, pos, g_q=g_q, g_k=g_k, n_new=n_new)
    h.qk_norm_rope(q, k, q, k, rope, pos, g_q=g_q, g_k=g_k, n_new=n_new)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    h.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("page,layout", [(1, "heads_first"), (16, "rows_first"), (24, "interleaved")])
@pytest.mark.parametrize("B,n,gains", [(1, 1, True), (4, 33, True), (5, 3, False)])
def test_append(pkg, dtype, Hq, Hkv, D, page, layout, B, n, gains):
    q, k, v, g_q, g_k, pos, n_new, rope = rows_case(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, B=B, n=n, gains=gains, seed=page)
    g = rng(4)
    pages = -(-(40 + n) // page)
    n_pages, table = tables(g, B, pages)
    kp, vp = pool(g, n_pages, Hkv, page, D, DT[dtype], layout)
    w = torch.rand(n_pages, Hkv, page, generator=g, device="cuda")
    kv_len = torch.randint(0, 41, (B,), generator=g, device="cuda", dtype=torch.int32)
    h = handle(pkg, Hq, Hkv, D, dtype, page_size=page, max_batch=B, max_pages=pages)
    cache = h.cache(kp, vp, table, kv_len, weights=w)
    want_k, want_v, want_w, tol = kp.double(), vp.double(), w.clone(), torch.zeros(kp.shape, dtype=torch.float64, device="cuda")
    qo = torch.full((B, n, Hq, D), 7.0, dtype=DT[dtype], device="cuda")
    h.append(cache, q, k, v, qo, rope, g_q=g_q, g_k=g_k, pos=pos, n_new=n_new)
    assert h.status() == 0
    for b in range(B):
        m, L = int(n_new[b]), int(kv_len[b])
        y, t = ref.norm_rope(q[b, :m], g_q, rope, int(pos[b]), EPS)
        ref.within(qo[b, :m], y, t + bf16_more(dtype, y), "q")
        assert (qo[b, m:] == 7.0).all()
        y, t = ref.norm_rope(k[b, :m], g_k, rope, int(pos[b]), EPS)
        for i in range(m):
            at, off = int(table[b, (L + i) // page]), (L + i) % page
            want_k[at, :, off], tol[at, :, off] = y[i], t[i] + bf16_more(dtype, y[i])
            want_v[at, :, off] = v[b, i].double()
            want_w[at, :, off] = 0
    ref.within(kp, want_k, tol, "k pages")                  # all other rows bit for bit
    assert torch.equal(vp.double(), want_v) and torch.equal(w, want_w)
    h.close()


FEW = [(2, 1, 64), (4, 4, 64), (1, 1, 64), (3, 1, 64), (6, 2, 64), (8, 2, 128), (1, 1, 128), (5, 1, 128), (7, 7, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", FEW)
@pytest.mark.parametrize("B,n,order", [(37, 701, "fused"), (300, 37, "heads")])
def test_norm_rope_and_gradient_of_few_heads(pkg, dtype, Hq, Hkv, D, B, n, order):
    """Rows enough that a warp takes several at a time, of one sequence or of two, some past n_new."""
    test_norm_rope_and_gradient(pkg, dtype, Hq, Hkv, D, order == "fused", B, n, order)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", FEW)
def test_append_few_heads(pkg, dtype, Hq, Hkv, D):
    test_append(pkg, dtype, Hq, Hkv, D, 24, "rows_first", 19, 301, True)


def test_append_positions_default_to_slots(pkg):
    q, k, v, _, _, _, _, rope = rows_case(pkg, Hq=4, Hkv=4, D=64, dtype="f32", B=2, n=3, gains=False)
    h = handle(pkg, 4, 4, 64, "f32", max_batch=2, max_pages=2)
    kp, vp = (torch.zeros(4, 4, 16, 64, device="cuda") for _ in range(2))
    table = torch.tensor([[3, 1], [0, 2]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([14, 0], dtype=torch.int32, device="cuda")
    qo, qo2 = torch.empty(2, 3, 4, 64, device="cuda"), torch.empty(2, 3, 4, 64, device="cuda")
    cache = h.cache(kp, vp, table, kv_len)
    h.append(cache, q, k, v, qo, rope)
    first = kp.clone()
    h.append(cache, q, k, v, qo2, rope, pos=kv_len.clone())
    assert torch.equal(qo, qo2) and torch.equal(kp, first) and kv_len.tolist() == [14, 0]
    h.close()


@pytest.mark.parametrize("what,bit", [("slot", 2), ("page", 16), ("n_new", 4), ("position", 32), ("negative", 32)])
def test_append_device_flags(pkg, what, bit):
    q, k, v, _, _, pos, n_new, rope = rows_case(pkg, Hq=4, Hkv=4, D=64, dtype="bf16", B=2, n=3, gains=False)
    h = handle(pkg, 4, 4, 64, "bf16", max_batch=2, max_pages=2)
    kp, vp = (torch.zeros(4, 4, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.tensor([[3, 1], [0, 2]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    n_new = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    if what == "slot":
        kv_len[1] = 31
    elif what == "page":
        table[1, 0] = -1
    elif what == "n_new":
        n_new[1] = 4
    else:
        pos[1] = rope.shape[0] - 1 if what == "position" else -1
    qo = torch.empty(2, 3, 4, 64, device="cuda", dtype=torch.bfloat16)
    h.append(h.cache(kp, vp, table, kv_len), q, k, v, qo, rope, pos=pos, n_new=n_new)
    assert h.status() == bit
    y, t = ref.norm_rope(k[0], None, rope, 0, EPS)
    ref.within(kp[3, :, :3].transpose(0, 1), y, t + 2.0 ** -8 * y.abs())   # the other sequence's rows are in place
    if what == "slot":
        assert torch.equal(vp[2, :, 15], v[1, 0]) and (vp[1] == 0).all()
    if what == "page":
        assert (kp[0] == 0).all() and (kp[2] == 0).all()
    h.close()


# ------------------------------------------------------------------- eviction

def check_evict(pkg, *, Hkv, D, dtype, page, lens, budget, sinks, recent, weights="mixed", pools="one", layout="heads_first",
                alias_len=False, seed=0, spare_pages=0):
    g, B, dt = rng(seed), len(lens), DT[dtype]
    pages, to_pages = -(-max(max(lens), 1) // page) + spare_pages, -(-budget // page)
    n = B * (pages + to_pages)
    perm = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(B, -1)
    table, table_to = perm[:, :pages].contiguous(), perm[:, pages:].contiguous()
    k, v = pool(g, n, Hkv, page, D, dt, layout)
    w = torch.rand(n, Hkv, page, generator=g, device="cuda")
    if weights == "ties":
        w = torch.floor(w * 4) / 4
        w[w == 0.25] = -0.0
        w[w == 0.5] = 0.0
    elif weights == "same":
        w.fill_(0.125)
    elif weights == "wild":
        r = torch.rand(w.shape, generator=g, device="cuda")
        w[r < 0.2] = math.nan
        w[r > 0.8] = math.inf
        w[(r > 0.7) & (r < 0.8)] = -math.inf
        w[(r > 0.5) & (r < 0.6)] *= -1
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    h = handle(pkg, Hkv, Hkv, D, dtype, page_size=page, max_batch=B, max_pages=max(pages, to_pages))
    src = h.cache(k, v, table, kv_len, weights=w)
    k2, v2, w2 = (k, v, w) if pools == "one" else (*pool(g, n, Hkv, page, D, dt, "rows_first"), torch.full_like(w, 9.0))
    len_to = kv_len if alias_len else torch.full_like(kv_len, -5)
    dst = h.cache(k2, v2, table_to, len_to, weights=None if pools == "no_weights" else w2)
    kept = torch.full((B, Hkv, budget), 77, dtype=torch.int32, device="cuda")
    before = [t.clone() for t in (k, v, w, k2, v2, w2)]
    h.evict(src, dst, kept, sinks=sinks, recent=recent)
    assert h.status() == 0
    assert len_to.tolist() == [min(x, budget) for x in lens]
    want = [t.clone() for t in before[3:]]
    tab, tab2 = table.cpu().long(), table_to.cpu().long()
    for b, L in enumerate(lens):
        wb = ref.gather(before[2], tab[b], L).cpu().numpy()
        for hd in range(Hkv):
            rows = ref.kept_rows(wb[hd], L, budget, sinks, recent)
            got = kept[b, hd].cpu().numpy()
            assert np.array_equal(got[:len(rows)], rows) and (got[len(rows):] == -1).all()
            j = torch.arange(len(rows))
            rows = torch.from_numpy(rows)
            for i in range(3):
                want[i][tab2[b, j // page], hd, j % page] = before[i][tab[b, rows // page], hd, rows % page]
    for i, (a, t) in enumerate(zip((k2, v2, w2), want)):
        if i == 2 and pools == "no_weights":
            t = before[5]
        assert torch.equal(torch.nan_to_num(a.float(), nan=123.0), torch.nan_to_num(t.float(), nan=123.0)), i
    h.close()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("weights", ["mixed", "ties", "same", "wild"])
@pytest.mark.parametrize("page,budget,sinks,recent", [(16, 64, 4, 20), (5, 33, 0, 0), (24, 100, 60, 40), (1, 1, 0, 0), (16, 1, 1, 0)])
def test_evict(pkg, dtype, D, weights, page, budget, sinks, recent):
    check_evict(pkg, Hkv=3, D=D, dtype=dtype, page=page, lens=[0, 1, budget, budget + 1, 3 * budget + 37], budget=budget, sinks=sinks,
                recent=recent, weights=weights)


@pytest.mark.parametrize("pools", ["one", "two", "no_weights"])
@pytest.mark.parametrize("layout", ["heads_first", "rows_first", "interleaved"])
def test_evict_pools_layouts_and_aliased_lengths(pkg, pools, layout):
    check_evict(pkg, Hkv=2, D=128, dtype="bf16", page=16, lens=[300, 77, 5], budget=90, sinks=3, recent=17, pools=pools, layout=layout,
                alias_len=True, spare_pages=2)


@pytest.mark.parametrize("weights", ["mixed", "same", "wild"])
@pytest.mark.parametrize("L", [5000, 49152 + 10, 60001])
def test_evict_long_rows(pkg, weights, L):
    check_evict(pkg, Hkv=1, D=64, dtype="bf16", page=64, lens=[L, 1200], budget=1111, sinks=5, recent=99, weights=weights)


def test_evict_budget_above_every_length(pkg):
    check_evict(pkg, Hkv=2, D=64, dtype="f32", page=16, lens=[30, 0, 64], budget=90, sinks=3, recent=17)


def test_evict_reports_bad_pages(pkg):
    h = handle(pkg, 2, 2, 64, "f32", max_batch=1, max_pages=4)
    k, v, w = torch.zeros(8, 2, 16, 64, device="cuda"), torch.zeros(8, 2, 16, 64, device="cuda"), torch.rand(8, 2, 16, device="cuda")
    table, to = torch.tensor([[0, 1, 99, 3]], dtype=torch.int32, device="cuda"), torch.tensor([[4, -1]], dtype=torch.int32, device="cuda")
    n = torch.tensor([60], dtype=torch.int32, device="cuda")
    kept = torch.empty(1, 2, 32, dtype=torch.int32, device="cuda")
    h.evict(h.cache(k, v, table, n, weights=w), h.cache(k, v, to, torch.zeros_like(n), weights=w), kept)
    assert h.status() == 16
    h.close()


# --------------------------------------------------------------- together

def test_decode_steps_in_a_graph_with_eviction(pkg):
    """Append, attention and eviction over many tokens against a plain 64-bit model of
    the whole loop; the step is captured once as a CUDA graph."""
    B, Hq, Hkv, D, page, budget, slack, prompt = 3, 8, 2, 64, 16, 48, 8, 30
    g = rng(11)
    pages = -(-(budget + slack) // page)
    n = 2 * B * pages
    perm = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(2, B, pages).contiguous()
    k, v, w = torch.zeros(n, Hkv, page, D, device="cuda"), torch.zeros(n, Hkv, page, D, device="cuda"), torch.zeros(n, Hkv, page, device="cuda")
    h = handle(pkg, Hq, Hkv, D, "f32", page_size=page, max_batch=B, max_pages=pages, track_weights=True)
    kv_len, pos = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    caches = [h.cache(k, v, perm[i], kv_len, weights=w) for i in range(2)]
    rope = pkg.rope_table(200, D)
    kept = torch.empty(B, Hkv, budget, dtype=torch.int32, device="cuda")
    g_q, g_k = (normal(g, D, dtype=torch.float32, scale=0.1) + 1 for _ in range(2))
    x = normal(g, B, 1, (Hq + 2 * Hkv) * D, dtype=torch.float32)
    q, kk, vv = (t.unflatten(-1, (-1, D)) for t in x.split([Hq * D, Hkv * D, Hkv * D], -1))
    qo, out = torch.empty(B, 1, Hq, D, device="cuda"), torch.empty(B, Hq, D, device="cuda")

    def step(c):
        h.append(c, q, kk, vv, qo, rope, g_q=g_q, g_k=g_k, pos=pos)
        h.attend(c, qo.view(B, Hq, D), out)
        kv_len.add_(1)
        pos.add_(1)

    # the 64-bit model: lists of rows per (sequence, KV head)
    rows = [[dict(k=[], v=[], w=[]) for _ in range(Hkv)] for _ in range(B)]
    xp = normal(g, B, prompt, (Hq + 2 * Hkv) * D, dtype=torch.float32)
    pq, pk, pv = (t.unflatten(-1, (-1, D)) for t in xp.split([Hq * D, Hkv * D, Hkv * D], -1))
    n_new = torch.tensor([prompt, 11, 1], dtype=torch.int32, device="cuda")
    h.append(caches[0], pq, pk, pv, torch.empty(B, prompt, Hq, D, device="cuda"), rope, g_q=g_q, g_k=g_k, pos=pos, n_new=n_new)
    for b in range(B):
        y = ref.norm_rope(pk[b, :int(n_new[b])], g_k, rope, 0, EPS)[0]
        for i in range(int(n_new[b])):
            for hd in range(Hkv):
                r = rows[b][hd]
                r["k"].append(y[i, hd]), r["v"].append(pv[b, i, hd].double()), r["w"].append(0.0)
    kv_len.add_(n_new)
    pos.add_(n_new)

    graphs, at = {}, 0
    for t in range(60):
        x.copy_(normal(g, B, 1, (Hq + 2 * Hkv) * D, dtype=torch.float32))
        if at not in graphs:
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                step(caches[at])
            graphs[at] = graph
        p0 = pos.tolist()
        graphs[at].replay()
        for b in range(B):
            qr, kr = (ref.norm_rope(a[b], gain, rope, p0[b], EPS)[0][0] for a, gain in ((q, g_q), (kk, g_k)))
            for hd in range(Hkv):
                r = rows[b][hd]
                r["k"].append(kr[hd]), r["v"].append(vv[b, 0, hd].double()), r["w"].append(0.0)
                z = qr[hd * 4:hd * 4 + 4] @ torch.stack(r["k"]).T * D ** -0.5
                p = torch.softmax(z, 1)
                want = p @ torch.stack(r["v"])
                assert (out[b, hd * 4:hd * 4 + 4].double() - want).abs().max() < 1e-4 * want.abs().max() + 1e-5
                r["w"] = [a + c for a, c in zip(r["w"], p.sum(0).tolist())]
        if int(kv_len.max()) == budget + slack:
            h.evict(caches[at], caches[1 - at], kept, sinks=2, recent=8)
            at = 1 - at
            for b in range(B):
                for hd in range(Hkv):
                    r = rows[b][hd]
                    keep = [i for i in kept[b, hd].tolist() if i >= 0]      # held to the formula's choice by weight
                    L = len(r["w"])
                    assert keep[:2] == [0, 1] and keep == sorted(set(keep)) and len(keep) == min(L, budget)
                    if L > budget:
                        assert set(range(L - 8, L)) <= set(keep)
                        left = [r["w"][i] for i in range(L) if i not in set(keep)]
                        mid = [r["w"][i] for i in keep if 2 <= i < L - 8]
                        assert min(mid) >= max(left) - 1e-4
                    for f in r:
                        r[f] = [r[f][i] for i in keep]
    assert h.status() == 0
    h.close()


# ----------------------------------------------------------------- refusals

def test_refusals(pkg):
    h = handle(pkg, 8, 2, 64, "bf16", max_batch=2, max_pages=4)
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    mk = lambda *s, dt=bf: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    k, v, w = mk(9, 2, 16, 64), mk(9, 2, 16, 64), mk(9, 2, 16, dt=f32)
    table, n = mk(2, 4, dt=i32), mk(2, dt=i32)
    q, out = mk(2, 8, 64), mk(2, 8, 64)
    cache = h.cache(k, v, table, n)
    for args in ((k.float(), v, table, n), (k, v[:, :, :8], table, n), (k, v.transpose(2, 3).contiguous().transpose(2, 3), table, n),
                 (k, v, table.long(), n), (k, v, table, n[:1]), (k, v, table[:, ::2], n), (k, v, table.cpu(), n),
                 (mk(9, 2, 16, 128)[..., ::2],) * 2 + (table, n)):
        with pytest.raises(ValueError):
            h.cache(*args)
    with pytest.raises(ValueError):
        h.cache(k, v, table, n, weights=w[:, :, :4])
    with pytest.raises(pkg.PrismError, match="track_weights"):
        h.attend(h.cache(k, v, table, n, weights=w), q, out)
    with pytest.raises(pkg.PrismError, match="CAPACITY"):
        h.attend(h.cache(k, v, mk(3, 4, dt=i32), mk(3, dt=i32)), mk(3, 8, 64), mk(3, 8, 64))
    with pytest.raises(pkg.PrismError, match="CAPACITY"):
        h.attend(h.cache(k, v, mk(2, 5, dt=i32), n), q, out)
    with pytest.raises(pkg.PrismError, match="16 bytes"):
        odd = mk(9 * 2 * 16 * 64 + 4)[4:].view(9, 2, 16, 64)
        h.attend(h.cache(odd, odd, table, n), q, out)
    with pytest.raises(pkg.PrismError, match="INVALID_ARG"):
        h.attend(cache, q, out, added=-1)
    for bad in ((mk(2, 8, 128)[..., ::2], out), (q, out[:1]), (q.float(), out), (q, out.cpu())):
        with pytest.raises(ValueError):
            h.attend(cache, *bad)
    with pytest.raises(TypeError):
        h.attend(None, q, out)
    other = handle(pkg, 8, 2, 64, "bf16", page_size=32, max_batch=2, max_pages=4)
    with pytest.raises(ValueError):
        other.attend(cache, q, out)
    q4, k4, rope, pos = mk(2, 3, 8, 64), mk(2, 3, 2, 64), pkg.rope_table(8, 64), mk(2, dt=i32)
    gain = mk(64)
    with pytest.raises(pkg.PrismError, match="together"):
        h.append(cache, q4, k4, k4, mk(2, 3, 8, 64), rope, g_q=gain)
    with pytest.raises(pkg.PrismError, match="only then"):
        h.qk_norm_rope_backward(q4, k4, q4, k4, mk(2, 3, 8, 64), mk(2, 3, 2, 64), rope, pos, g_q=gain, g_k=gain)
    with pytest.raises(pkg.PrismError, match="null"):
        h.qk_norm_rope(q4, k4, mk(2, 3, 8, 64), mk(2, 3, 2, 64), rope, None)
    with pytest.raises(pkg.PrismError, match="16 bytes"):
        h.append(cache, q4, mk(2, 3, 2, 68)[..., 2:66], k4, mk(2, 3, 8, 64), rope)
    with pytest.raises(ValueError):
        h.append(cache, q4, k4, k4, mk(2, 3, 8, 64), rope[:, :, :16])
    with pytest.raises(ValueError):
        h.append(cache, q4[:1], k4, k4, mk(2, 3, 8, 64), rope)
    src = h.cache(k, v, table, n, weights=w)
    dst = h.cache(k, v, mk(2, 1, dt=i32), mk(2, dt=i32), weights=w)
    kept = lambda b: mk(2, 2, b, dt=i32)  # noqa: E731
    with pytest.raises(pkg.PrismError, match="SHAPE"):
        h.evict(src, dst, kept(17))
    with pytest.raises(pkg.PrismError, match="sinks"):
        h.evict(src, dst, kept(16), sinks=9, recent=8)
    with pytest.raises(pkg.PrismError, match="sinks"):
        h.evict(src, dst, kept(16), sinks=-1)
    with pytest.raises(pkg.PrismError, match="block table"):
        h.evict(src, src, kept(16))
    with pytest.raises(pkg.PrismError, match="weights"):
        h.evict(cache, dst, kept(16))
    with pytest.raises(ValueError):
        h.evict(src, dst, mk(2, 3, 16, dt=i32))
    assert h.status() == 0
    for bad in (dict(head_dim=96), dict(n_kv_heads=3), dict(page_size=0), dict(max_batch=0), dict(max_pages=2 ** 30, page_size=64),
                dict(rms_eps=-1.0), dict(softmax_scale=float("nan"))):
        with pytest.raises(pkg.PrismError):
            handle(pkg, 8, 2, 64, "bf16", **bad)
    with pytest.raises(ValueError):
        handle(pkg, 8, 2, 64, "f16")


# ------------------------------------------------- work divided over many CTAs

@pytest.mark.parametrize("Hq,D,dtype,n", [(4, 128, "bf16", 70001), (8, 128, "bf16", 50003), (16, 128, "bf16", 45007), (16, 64, "bf16", 60000),
                                          (1, 64, "bf16", 90001), (4, 64, "f32", 30011), (8, 128, "f32", 20005)])
def test_attend_one_segment_over_the_whole_gpu(pkg, Hq, D, dtype, n):
    """One KV head: its rows are cut over every CTA, joined in groups, then the groups."""
    check_attend(pkg, Hq=Hq, Hkv=1, D=D, dtype=dtype, page=64, lens=[n], track=True, wild=False)


def test_attend_long_among_short(pkg):
    check_attend(pkg, Hq=16, Hkv=1, D=128, dtype="bf16", page=32, lens=[3, 40000, 0, 1, 64, 65, 12000] + [17] * 20, track=True, wild=False)
    check_attend(pkg, Hq=8, Hkv=2, D=64, dtype="f32", page=16, lens=[5] * 40 + [9000] + [5] * 40, wild=False)


def test_evict_rows_beyond_shared_memory(pkg):
    """More rows than eight CTAs' shared memory holds the keys of."""
    check_evict(pkg, Hkv=1, D=64, dtype="bf16", page=128, lens=[400100], budget=3001, sinks=7, recent=500)
    check_evict(pkg, Hkv=1, D=64, dtype="bf16", page=128, lens=[400100], budget=3001, sinks=7, recent=500, weights="same")


def test_evict_many_short_sequences(pkg):
    check_evict(pkg, Hkv=8, D=64, dtype="bf16", page=16, lens=[60 + 7 * (i % 13) for i in range(50)], budget=75, sinks=2, recent=9)
    check_evict(pkg, Hkv=40, D=64, dtype="bf16", page=64, lens=[2500 + i for i in range(9)], budget=900, sinks=2, recent=9, weights="ties")


def test_example_bounds_the_cache(pkg):
    """The decode example: caches within budget + slack (evictions before tokens 31, 51 and 71), every kept row a row of the past, finite results."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    layer, evictions = example.main(["--batch", "3", "--prompt", "300", "--tokens", "90", "--budget", "310", "--slack", "20", "--hidden", "256"])
    assert evictions == 3 and int(layer.kv_len.max()) <= 330 and int(layer.pos.max()) == 390
    assert torch.isfinite(layer.y.float()).all()
    h, B = layer.caches[layer.at], layer.B
    for b in range(B):                       # weights of the kept rows: each row got at most one unit per query head and step
        n = int(layer.kv_len[b])
        w = ref.gather(layer.weights, h.block_table[b].cpu(), n)
        assert (w >= 0).all() and float(w.max()) <= 4 * 90 + 1e-3
    layer.att.close()


@pytest.mark.parametrize("what,bit", [("long", 2), ("negative", 2)])
def test_evict_device_flags(pkg, what, bit):
    """A length outside the table: clamped and reported; the other sequence as it should be."""
    h = handle(pkg, 2, 2, 64, "f32", max_batch=2, max_pages=3)
    k, v, w = torch.randn(12, 2, 16, 64, device="cuda"), torch.randn(12, 2, 16, 64, device="cuda"), torch.rand(12, 2, 16, device="cuda")
    table = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32, device="cuda")
    to = torch.tensor([[6, 7], [8, 9]], dtype=torch.int32, device="cuda")
    n = torch.tensor([40, 49 if what == "long" else -2], dtype=torch.int32, device="cuda")
    out, kept = torch.zeros_like(n), torch.empty(2, 2, 20, dtype=torch.int32, device="cuda")
    h.evict(h.cache(k, v, table, n, weights=w), h.cache(k, v, to, out, weights=w), kept, sinks=1, recent=3)
    assert h.status() == bit
    assert out.tolist() == [20, 20 if what == "long" else 0]
    for hd in range(2):
        wl = ref.gather(w, table[0].cpu(), 40)[hd].cpu().numpy()
        assert np.array_equal(kept[0, hd].cpu().numpy(), ref.kept_rows(wl, 40, 20, 1, 3))
        assert (kept[1, hd] == -1).all() == (what == "negative")
    h.close()


@pytest.mark.parametrize("what,bit", [("n_new", 4), ("position", 32)])
def test_gradient_device_flags(pkg, what, bit):
    q, k, _, g_q, g_k, pos, _, rope = rows_case(pkg, Hq=4, Hkv=2, D=64, dtype="f32", B=2, n=3, gains=True)
    pos, n_new = torch.tensor([0, 5], dtype=torch.int32, device="cuda"), torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    if what == "n_new":
        n_new[1] = -1
    else:
        pos[1] = rope.shape[0]
    h = handle(pkg, 4, 2, 64, "f32")
    g = rng(3)
    dqo, dko = normal(g, 2, 3, 4, 64, dtype=torch.float32), normal(g, 2, 3, 2, 64, dtype=torch.float32)
    dq, dk, dg = torch.empty_like(dqo), torch.empty_like(dko), torch.empty(2, 64, device="cuda")
    h.qk_norm_rope_backward(dqo, dko, q, k, dq, dk, rope, pos, g_q=g_q, g_k=g_k, dg_q=dg[0], dg_k=dg[1], n_new=n_new)
    assert h.status() == bit
    want, _, tol, _ = ref.norm_rope_grad(q[0], g_q, dqo[0], rope, 0, EPS)
    ref.within(dq[0], want, tol)
    if what == "n_new":
        assert (dq[1] == 0).all() and (dk[1] == 0).all()
    h.close()


def test_broadcast_inputs_and_overlapping_outputs(pkg):
    """One row for every sequence, one key head for every KV head (strides of 0) as inputs: as their copies.  As outputs: refused."""
    B, n, Hq, Hkv, D = 3, 4, 8, 2, 64
    g = rng(8)
    q1, k1 = normal(g, 1, n, Hq, D, dtype=torch.bfloat16), normal(g, B, n, 1, D, dtype=torch.bfloat16)
    q, k = q1.expand(B, n, Hq, D), k1.expand(B, n, Hkv, D)
    dy, dk_out = normal(g, B, n, Hq, D, dtype=torch.bfloat16), normal(g, 1, 1, Hkv, D, dtype=torch.bfloat16).expand(B, n, Hkv, D)
    pos, rope = torch.tensor([0, 3, 9], dtype=torch.int32, device="cuda"), pkg.rope_table(20, D)
    gains = [normal(g, D, dtype=torch.bfloat16) for _ in range(2)]
    h = handle(pkg, Hq, Hkv, D, "bf16")
    got = []
    for a, b, c, d in ((q, k, dy, dk_out), (q.contiguous(), k.contiguous(), dy, dk_out.contiguous())):
        o = [torch.empty(B, n, H, D, dtype=torch.bfloat16, device="cuda") for H in (Hq, Hkv, Hq, Hkv)] + [torch.empty(2, D, device="cuda")]
        h.qk_norm_rope(a, b, o[0], o[1], rope, pos, g_q=gains[0], g_k=gains[1])
        h.qk_norm_rope_backward(c, d, a, b, o[2], o[3], rope, pos, g_q=gains[0], g_k=gains[1], dg_q=o[4][0], dg_k=o[4][1])
        got.append(o)
    assert all(torch.equal(x, y) for x, y in zip(*got))
    wide = torch.empty(1, n, Hq, D, dtype=torch.bfloat16, device="cuda").expand(B, n, Hq, D)
    with pytest.raises(pkg.PrismError, match="stride is 0"):
        h.qk_norm_rope(q, k, wide, got[0][1], rope, pos)
    with pytest.raises(pkg.PrismError, match="stride is 0"):
        h.qk_norm_rope_backward(dy, dk_out, q, k, wide, got[0][3], rope, pos)
    one = torch.empty(1, Hkv, 16, D, dtype=torch.bfloat16, device="cuda").expand(4, Hkv, 16, D)
    with pytest.raises(pkg.PrismError, match="stride is 0"):
        h.attend(h.cache(one, one, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")),
                 got[0][0][:1, 0].contiguous(), got[0][2][:1, 0].contiguous())
    h.close()


def test_gradient_of_tiny_rows(pkg):
    """Rows of 1e-18 without an epsilon: r is 1e18 and its powers are not, the gradient is."""
    Hq, Hkv, D = 4, 2, 64
    q, k, _, g_q, g_k, pos, _, rope = rows_case(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype="f32", B=1, n=3, gains=True)
    q, k = q * 1e-18, k * 1e-18
    h = handle(pkg, Hq, Hkv, D, "f32", rms_eps=0.0)
    g = rng(3)
    dqo, dko = normal(g, 1, 3, Hq, D, dtype=torch.float32), normal(g, 1, 3, Hkv, D, dtype=torch.float32)
    dq, dk, dg = torch.empty_like(dqo), torch.empty_like(dko), torch.empty(2, D, device="cuda")
    h.qk_norm_rope_backward(dqo, dko, q, k, dq, dk, rope, pos, g_q=g_q, g_k=g_k, dg_q=dg[0], dg_k=dg[1])
    for x, gain, dy, dx, dgain in ((q, g_q, dqo, dq, dg[0]), (k, g_k, dko, dk, dg[1])):
        want, dgw, tol, dgt = ref.norm_rope_grad(x[0], gain, dy[0], rope, int(pos[0]), 0.0)
        ref.within(dx[0], want, tol, "dx")
        ref.within(dgain, dgw, dgt, "dg")
    h.close()
