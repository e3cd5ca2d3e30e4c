"""The paged cache held in 8 bits on the GPU against its 64-bit forms (codes_ref.py):
rows quantised as they are written, read back, attended to."""
from __future__ import annotations

import math

import pytest
import torch

from . import codes_ref as ref
from . import paged_ref
from .paged_ref import U, within

pytestmark = pytest.mark.gpu
EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def pkg():
    import paper_2602_01762_gb300 as p
    return p


def rng(seed):
    return torch.Generator().manual_seed(seed)


def code_pool(g, n_pages, Hkv, page, D, fmt, r, layout="heads_first", spread=3):
    """Pages of codes in one of a program's storage orders, and their blocks' scales, powers of two or not."""
    def one():
        y = torch.randn(n_pages, Hkv, page, D, generator=g) * (110 if fmt == "e4m3" else 35)
        y = y.clamp(-ref.MOST[fmt], ref.MOST[fmt])
        return y.to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().to(torch.int8)
    def put(x):
        x = x.cuda()
        if layout == "heads_first":
            return x
        raw = x.view(torch.uint8)
        return raw.transpose(1, 2).contiguous().view(x.dtype).transpose(1, 2)
    unit = 2.0 ** -7 if fmt == "e4m3" else 2.0 ** -5
    scales = [unit * torch.exp2(torch.rand(n_pages, Hkv, page // r, generator=g) * 2 * spread - spread) for _ in range(2)]
    if layout == "interleaved":
        both = torch.stack([one(), one()], 1).cuda()
        return both[:, 0], both[:, 1], scales[0].cuda(), scales[1].cuda()
    return put(one()), put(one()), scales[0].cuda(), scales[1].cuda()


def tables(g, B, pages, spare=3):
    n = B * pages + spare
    return n, torch.randperm(n, generator=g).to(torch.int32)[:B * pages].view(B, pages).contiguous()


def setup(pkg, *, Hq, Hkv, D, dtype, fmt, page, r, lens, layout="heads_first", scale=None, seed=0, qscale=1.5, room=1, wild=True, spread=3):
    g = rng(seed)
    B = len(lens)
    pages = max(1, -(-max(lens) // page)) + room
    n_pages, table = tables(g, B, pages)
    k, v, ks, vs = code_pool(g, n_pages, Hkv, page, D, fmt, r, layout, spread)
    owned = table.clone()
    if wild:                             # entries past a sequence's rows are never followed; scales nobody's rows have are NaN
        used = torch.zeros(n_pages, page // r, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(0, n):
                used[int(table[b, j // page]), j % page // r] = True
            table[b, -(-n // page):] = -7 if b % 2 else 2 ** 31 - 1
        for s in (ks, vs):
            s.masked_fill_(~used.cuda()[:, None], float("nan"))
    q = (torch.randn(B, Hq, D, generator=g) * qscale).to(DT[dtype]).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((B, Hq), 7.0, device="cuda")
    h = pkg.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=B, max_pages=pages,
                           softmax_scale=scale, rms_eps=EPS)
    cache = h.cache(k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), k_scales=ks, v_scales=vs)
    return h, cache, q, out, lse, scale if scale is not None else D ** -0.5, owned


def check_attend(pkg, window=None, sinks=0, **kw):
    h, cache, q, out, lse, scale, owned = setup(pkg, **kw)
    if window is not None:               # entries of pages without a seen row are never followed, scales without one never read
        page, table = kw["page"], cache.block_table.cpu()
        seen = torch.zeros(cache.k_scales.shape[0], page, dtype=torch.bool)
        for b, n in enumerate(kw["lens"]):
            j = ref.seen(n, window, sinks)
            seen[owned[b].long()[j // page], j % page] = True
            table[b][~seen[owned[b].long()].any(1)] = -5 if b % 2 else 2 ** 31 - 1
        cache.block_table.copy_(table)
        lost = ~seen.view(seen.shape[0], -1, kw["r"]).any(2).cuda()
        for s in (cache.k_scales, cache.v_scales):
            s.masked_fill_(lost[:, None], float("nan"))
    h.attend(cache, q, out, lse=lse, added=0, window=window, sinks=sinks)
    assert h.status() == 0
    k, v = ref.values(cache.k_pages, cache.k_scales), ref.values(cache.v_pages, cache.v_scales)
    o, l, _, to, tl, _ = ref.attend(q, k, v, owned, kw["lens"], scale, window, sinks, cache.v_scales.cpu())
    within(out.cpu(), o, to, "out")
    within(lse.cpu(), l, tl, "lse")
    first = out.clone()
    h.attend(cache, q, out, lse=lse, added=0, window=window, sinks=sinks)
    assert torch.equal(out, first)       # the same bits again
    h.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (6, 2), (8, 2), (5, 1), (14, 2), (8, 1), (9, 1), (16, 1), (20, 1), (64, 2)])
def test_attend_groups(pkg, fmt, dtype, D, Hq, Hkv):
    check_attend(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, fmt=fmt, page=16, r=8, lens=[37, 300, 1])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("page,r", [(1, 1), (5, 1), (5, 5), (16, 16), (24, 6), (24, 24), (64, 2), (200, 100)])
@pytest.mark.parametrize("layout", ["heads_first", "rows_first", "interleaved"])
def test_attend_pages_blocks_and_layouts(pkg, fmt, page, r, layout):
    check_attend(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", fmt=fmt, page=page, r=r, lens=[0, 1, 15, 16, 17, 127, 128, 129, 395], layout=layout, seed=page)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 257])
def test_attend_lengths_around_tiles(pkg, D, n):
    for dtype in DT:
        for fmt in ref.MOST:
            check_attend(pkg, Hq=4, Hkv=1, D=D, dtype=dtype, fmt=fmt, page=8, r=8, lens=[n])


@pytest.mark.parametrize("B", [32, 33, 129, 300])
def test_attend_batches(pkg, B):
    lens = [(37 * i * i + 11) % 331 for i in range(B)]
    check_attend(pkg, Hq=8, Hkv=2, D=64, dtype="bf16", fmt="e4m3", page=16, r=4, lens=lens)
    check_attend(pkg, Hq=2, Hkv=2, D=64, dtype="f32", fmt="int8", page=16, r=1, lens=lens, wild=False)


@pytest.mark.parametrize("dtype,fmt,lens", [("bf16", "e4m3", [40007]), ("bf16", "int8", [9, 20011, 0, 4999]), ("f32", "e4m3", [9001])])
def test_attend_long_rows_are_joined(pkg, dtype, fmt, lens):
    check_attend(pkg, Hq=8, Hkv=2, D=128, dtype=dtype, fmt=fmt, page=64, r=32, lens=lens, wild=False)


@pytest.mark.parametrize("qscale", [0.0, 1e-3, 30.0, 1e-30, 1e30])
def test_attend_peaked_and_flat_scores(pkg, qscale):
    for dtype in DT:
        for Hq in (8, 16):
            check_attend(pkg, Hq=Hq, Hkv=2, D=128, dtype=dtype, fmt="int8", page=16, r=16, lens=[700, 90], qscale=qscale,
                         scale=None if qscale < 1e3 else 1e-30)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("spread", [20, 45])
def test_attend_scales_far_apart(pkg, fmt, spread):
    """V's blocks differ by up to 2^90, far beyond fp16: each row's weight keeps its bits."""
    for dtype in DT:
        for Hq in (4, 8, 16):
            h, cache, q, out, lse, scale, _ = setup(pkg, Hq=Hq, Hkv=1, D=64, dtype=dtype, fmt=fmt, page=16, r=8, lens=[431, 77], spread=spread)
            cache.k_scales.clamp_(max=2.0 ** -5)
            h.attend(cache, q, out, lse=lse, added=0)
            k, v = ref.values(cache.k_pages, cache.k_scales), ref.values(cache.v_pages, cache.v_scales)
            o, l, _, to, tl, _ = ref.attend(q, k, v, cache.block_table, [431, 77], scale, v_scales=cache.v_scales.cpu())
            within(out.cpu(), o, to, "out")
            within(lse.cpu(), l, tl, "lse")
            # and with the scales in order, growing or shrinking over the rows
            for order in (False, True):
                at = cache.block_table[0].cpu()
                for i in range(27):
                    cache.v_scales[int(at[i])] = 2.0 ** (2 * spread / 27 * (i if order else 26 - i) - spread)
                h.attend(cache, q, out, lse=lse, added=0)
                v = ref.values(cache.v_pages, cache.v_scales)
                o, _, _, to, _, _ = ref.attend(q[:1], k, v, cache.block_table[:1], [431], scale, v_scales=cache.v_scales.cpu())
                within(out[:1].cpu(), o, to, "ordered")
            h.close()


def test_attend_scales_of_zero_and_tiny_ones(pkg):
    for dtype in DT:
        h, cache, q, out, lse, scale, _ = setup(pkg, Hq=4, Hkv=1, D=64, dtype=dtype, fmt="int8", page=16, r=16, lens=[100], wild=False)
        cache.v_scales.zero_()
        h.attend(cache, q, out, lse=lse, added=0)
        assert (out == 0).all() and torch.isfinite(lse).all()
        cache.v_scales.fill_(2.0 ** -126)
        cache.v_pages.fill_(3)
        h.attend(cache, q, out, added=0)
        within(out.cpu(), torch.full(out.shape, 3 * 2.0 ** -126, dtype=torch.float64), torch.full(out.shape, 2.0 ** -134, dtype=torch.float64))
        cache.k_scales.zero_()           # every score 0: the mean, ln 100
        cache.v_scales.fill_(1.0)
        h.attend(cache, q, out, lse=lse, added=0)
        assert ((out.float() - 3).abs() <= 3 * 2.0 ** -8).all() and (lse - math.log(100)).abs().max() < 1e-5
        h.close()


def test_attend_nan_codes_and_scales(pkg):
    h, cache, q, out, lse, scale, _ = setup(pkg, Hq=8, Hkv=2, D=64, dtype="bf16", fmt="e4m3", page=16, r=16, lens=[50, 40], wild=False)
    h.attend(cache, q, out, lse=lse, added=0)
    was, was_lse = out.clone(), lse.clone()
    p = int(cache.block_table[0, 1])
    cache.v_pages.view(torch.uint8)[p, 1, 3, 9] = 0x7F
    h.attend(cache, q, out, lse=lse, added=0)
    bad = torch.zeros(2, 8, 64, dtype=torch.bool, device="cuda")
    bad[0, 4:, 9] = True
    assert torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], was[~bad]) and torch.equal(lse, was_lse)
    cache.k_scales[p, 0] = float("nan")
    h.attend(cache, q, out, lse=lse, added=0)
    assert torch.isnan(out[0, :4]).all() and torch.isnan(lse[0, :4]).all()
    assert torch.equal(out[1], was[1]) and torch.equal(lse[0, 4:], was_lse[0, 4:])
    h.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (0, 3), (16, 4), (64, 64), (100, 65), (129, 1), (333, 130), (1000, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_window_over_codes(pkg, fmt, window, sinks):
    for dtype, Hq, D in (("bf16", 4, 128), ("f32", 8, 64), ("bf16", 32, 64)):
        check_attend(pkg, Hq=Hq, Hkv=2, D=D, dtype=dtype, fmt=fmt, page=16, r=4, lens=[0, 1, 64, 65, 257, 700], window=window, sinks=sinks)


# ------------------------------------------------------------------ append

def identity_rope(n, D):
    t = torch.zeros(n, 2, D // 2)
    t[:, 0] = 1
    return t.cuda()


def append_case(pkg, *, D, dtype, fmt, page, r, lens, counts, Hq=4, Hkv=2, seed=0, grow=1.0, norm=False, layout="heads_first"):
    g = rng(seed)
    B, n = len(lens), max(max(counts), 1)
    pages = -(-(max(lens) + n) // page) + 1
    n_pages, table = tables(g, B, pages)
    k_pages, v_pages, ks, vs = code_pool(g, n_pages, Hkv, page, D, fmt, r, layout)
    ks, vs = (torch.exp2(torch.floor(torch.log2(s))) for s in (ks, vs))   # as an append leaves them
    q, k, v = (torch.randn(B, n, H, D, generator=g) for H in (Hq, Hkv, Hkv))
    size = grow ** torch.arange(n)[None, :, None, None]
    q, k, v = (x.to(DT[dtype]).cuda() for x in (q, k * size, v * size * 0.5))
    h = pkg.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=B, max_pages=pages, rms_eps=EPS)
    cache = h.cache(k_pages, v_pages, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), k_scales=ks, v_scales=vs)
    n_new = torch.tensor(counts, dtype=torch.int32).cuda()
    return h, cache, q, k, v, torch.zeros_like(q), n_new


def stored(cache, name, lens, x, counts, fmt):
    codes, scales = ref.codes_of(getattr(cache, name + "_pages")), getattr(cache, name + "_scales").cpu().double()
    ref.store(codes, scales, cache.block_table.cpu(), lens, x.cpu().double(), counts, fmt)
    return codes, scales


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page,r", [(1, 1), (8, 1), (16, 2), (16, 4), (24, 3), (24, 6), (16, 8), (16, 16), (64, 32), (96, 48), (128, 128), (200, 200)])
def test_append_is_exact(pkg, fmt, dtype, D, page, r):
    """No norm and no rotation: codes and scales are the formula's, bit for bit, those of
    earlier rows in a block that grows and of every row that is not touched too."""
    lens, counts = [0, 1, 5, 16, 33, 100], [37, 1, 2, 0, 18, 130]
    for grow in (1.0, 1.06):
        h, cache, q, k, v, q_out, n_new = append_case(pkg, D=D, dtype=dtype, fmt=fmt, page=page, r=r, lens=lens, counts=counts, grow=grow, seed=r)
        want = [stored(cache, n, lens, x, counts, fmt) for n, x in (("k", k), ("v", v))]
        h.append(cache, q, k, v, q_out, identity_rope(300, D), n_new=n_new)
        assert h.status() == 0
        for (codes, scales), name in zip(want, "kv"):
            assert torch.equal(getattr(cache, name + "_scales").cpu().double(), scales), name
            assert torch.equal(ref.codes_of(getattr(cache, name + "_pages")), codes), name
        for b, c in enumerate(counts):
            assert torch.equal(q_out[b, :c], q[b, :c]) and (q_out[b, c:] == 0).all()
        h.close()


@pytest.mark.parametrize("dtype,D,Hkv,page,r", [("bf16", 128, 1, 16, 16), ("bf16", 64, 1, 32, 32), ("bf16", 128, 5, 16, 8), ("f32", 64, 2, 32, 32),
                                                ("bf16", 128, 1, 16, 1), ("f32", 128, 3, 16, 2), ("bf16", 64, 1, 24, 3), ("bf16", 128, 1, 16, 4)])
def test_append_of_many_tiles(pkg, dtype, D, Hkv, page, r):
    """Prompts of more tiles than run at once, of which a CTA takes several: bit for bit, with lengths
    that end a sequence in its first tile, in the middle of a CTA's run of them and at its end."""
    n = 600 * r if r > 4 else 2048
    counts = [n, 3 * r + 1, 0, n - r, n - 2 * r - 1, 1, n - 5, n // 2]
    lens = [0, 1, 5, r - 1, 2 * r, 7, page, 3]
    h, cache, q, k, v, q_out, n_new = append_case(pkg, D=D, dtype=dtype, fmt="int8", page=page, r=r, lens=lens, counts=counts, Hq=Hkv, Hkv=Hkv, seed=r)
    want = [stored(cache, name, lens, x, counts, "int8") for name, x in (("k", k), ("v", v))]
    h.append(cache, q, k, v, q_out, identity_rope(n + 2 * page, D), n_new=n_new)
    assert h.status() == 0
    for (codes, scales), name in zip(want, "kv"):
        assert torch.equal(getattr(cache, name + "_scales").cpu().double(), scales), name
        assert torch.equal(ref.codes_of(getattr(cache, name + "_pages")), codes), name
    for b, c in enumerate(counts):
        assert torch.equal(q_out[b, :c], q[b, :c]) and (q_out[b, c:] == 0).all()
    h.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("page,r", [(16, 16), (24, 24), (64, 64), (100, 100), (128, 64)])
def test_append_one_token_anywhere_in_a_block(pkg, fmt, dtype, D, page, r):
    """A token behind 0 to r - 1 rows of its block: bit for bit, the earlier rows' codes too."""
    lens = list(range(0, 2 * r, max(r // 13, 1)))
    counts = [b % 7 > 0 for b in range(len(lens))]
    h, cache, q, k, v, q_out, n_new = append_case(pkg, D=D, dtype=dtype, fmt=fmt, page=page, r=r, lens=lens, counts=[int(c) for c in counts], Hq=4, Hkv=2, seed=r)
    want = [stored(cache, name, lens, x, [int(c) for c in counts], fmt) for name, x in (("k", k), ("v", v))]
    h.append(cache, q, k, v, q_out, identity_rope(2 * r + 2, D), n_new=n_new)
    assert h.status() == 0
    for (codes, scales), name in zip(want, "kv"):
        assert torch.equal(getattr(cache, name + "_scales").cpu().double(), scales), name
        assert torch.equal(ref.codes_of(getattr(cache, name + "_pages")), codes), name
    h.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("layout", ["rows_first", "interleaved"])
def test_append_to_other_layouts_token_by_token(pkg, fmt, layout):
    lens = [3, 16, 40]
    h, cache, q, k, v, q_out, _ = append_case(pkg, D=128, dtype="bf16", fmt=fmt, page=16, r=16, lens=lens, counts=[20] * 3, grow=1.1, layout=layout)
    for i in range(20):
        at = [n + i for n in lens]
        rows = [x[:, i:i + 1] for x in (q, k, v, q_out)]      # strided rows of a longer block
        want = [stored(cache, n, at, x, [1] * 3, fmt) for n, x in (("k", rows[1]), ("v", rows[2]))]
        h.append(cache, *rows, identity_rope(80, 128))
        for (codes, scales), name in zip(want, "kv"):
            assert torch.equal(getattr(cache, name + "_scales").cpu().double(), scales)
            assert torch.equal(ref.codes_of(getattr(cache, name + "_pages")), codes)
        cache.kv_len += 1
    assert h.status() == 0
    h.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 8, 2), ("f32", 64, 3, 3), ("bf16", 64, 16, 1), ("f32", 128, 8, 8)])
@pytest.mark.parametrize("gains", [False, True])
def test_append_norm_and_rotation(pkg, fmt, dtype, D, Hq, Hkv, gains):
    """Values within half a step of their block's scale and the norm's fp32 error of it,
    scales those of the largest value or, where that lies within its error of a border,
    of the next."""
    lens, counts, pos = [0, 7, 64], [50, 3, 20], [0, 9, 60]
    h, cache, q, k, v, q_out, n_new = append_case(pkg, D=D, dtype=dtype, fmt=fmt, page=16, r=8, lens=lens, counts=counts, Hq=Hq, Hkv=Hkv, seed=3)
    cache.k_scales.fill_(2.0 ** -20)     # earlier rows of no size: new scales show
    rope = pkg.rope_table(200, D, 10000.0)
    g = rng(9)
    g_q, g_k = ((torch.randn(D, generator=g) * 0.2 + 1).to(DT[dtype]).cuda() for _ in range(2)) if gains else (None, None)
    vals = stored(cache, "v", lens, v, counts, fmt)
    h.append(cache, q, k, v, q_out, rope, g_q=g_q, g_k=g_k, pos=torch.tensor(pos, dtype=torch.int32).cuda(), n_new=n_new)
    assert h.status() == 0
    assert torch.equal(ref.codes_of(cache.v_pages), vals[0]) and torch.equal(cache.v_scales.cpu().double(), vals[1])
    got, table = ref.values(cache.k_pages, cache.k_scales), cache.block_table.cpu()
    for b, (n, c) in enumerate(zip(lens, counts)):
        want_q, tol_q = paged_ref.norm_rope(q[b, :c], g_q, rope, pos[b], EPS)
        within(q_out[b, :c], want_q, tol_q + 2.0 ** -8 * want_q.abs() * (dtype == "bf16") + U * want_q.abs(), "q")
        want, tol = (x.cpu() for x in paged_ref.norm_rope(k[b, :c], g_k, rope, pos[b], EPS))
        for j in range(n // 8 * 8, n + c, 8):
            lo, hi = max(j, n), min(j + 8, n + c)
            p, row = int(table[b, j // 16]), j % 16
            for head in range(Hkv):
                x, t = want[lo - n:hi - n, head], tol[lo - n:hi - n, head]
                s = float(cache.k_scales[p, head, row // 8])
                top, off = float(x.abs().max()), float(t.max())
                assert s in (ref.scale_of(top - off, fmt), ref.scale_of(top + off, fmt))
                step = 0.5 if fmt == "int8" else torch.exp2((torch.frexp(x / s)[1] - 4).clamp(min=-9).double()) / 2
                slot = torch.arange(lo - j, hi - j) + row
                # a value at a border between two steps may take the larger one's half
                within(got[p, head, slot], x, t + 1.0001 * step * s * (2 if fmt == "e4m3" else 1), "k")
    h.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_extreme_values(pkg, fmt, dtype):
    """Zeros, the type's largest and smallest, NaN and infinities; a block that had a NaN
    scale, and one that starts afresh after it."""
    h, cache, q, k, v, q_out, _ = append_case(pkg, D=64, dtype=dtype, fmt=fmt, page=16, r=16, lens=[0] * 5, counts=[16] * 5, Hkv=1)
    big, inf, nan = torch.finfo(DT[dtype]).max, float("inf"), float("nan")
    k[0] = 0
    v[0] = -big
    k[1] = 1e-45
    k[1, 0, 0, 5] = 2.0 ** -126
    v[1, 3, 0, 7] = inf
    k[2, 2, 0, 1] = nan
    k[2, 3, 0, 2] = -inf
    h.append(cache, q, k, v, q_out, identity_rope(40, 64))
    assert h.status() == 0
    kv, vv = ref.values(cache.k_pages, cache.k_scales), ref.values(cache.v_pages, cache.v_scales)
    at = cache.block_table.cpu()[:, 0].long()
    assert (kv[at[0]] == 0).all() and float(cache.k_scales[at[0], 0, 0]) == 0.0
    assert (vv[at[0]].abs() / big - 1).abs().max() <= (2.0 ** -4 if fmt == "e4m3" else 2.0 ** -6)
    s = 2.0 ** -126
    assert float(cache.k_scales[at[1], 0, 0]) == s
    assert torch.equal(kv[at[1], 0], ref.nearest(k[1, :, 0].cpu().double() / s, fmt) * s)
    odd = torch.zeros(16, 64, dtype=torch.bool)
    if fmt == "int8":
        assert torch.isnan(vv[at[1]]).all() and torch.isnan(kv[at[2]]).all()
    else:
        odd[3, 7] = True
        assert torch.equal(torch.isnan(vv[at[1], 0]), odd)
        fine = torch.where(odd, 0.0, v[1, :, 0].cpu().double())
        assert torch.equal(vv[at[1], 0][~odd], (ref.nearest(fine / float(cache.v_scales[at[1], 0, 0]), fmt) * float(cache.v_scales[at[1], 0, 0]))[~odd])
        odd = torch.zeros(16, 64, dtype=torch.bool)
        # the rotation by an angle of 0 takes an infinity times 0 into the other half
        odd[2, 1] = odd[2, 33] = odd[3, 2] = odd[3, 34] = True
        assert torch.equal(torch.isnan(kv[at[2], 0]), odd)
    # one more row behind 15: a NaN scale stays; behind 0 the block starts afresh
    cache.kv_len.fill_(15)
    row = torch.ones_like(k[:, :1])
    h.append(cache, q[:, :1], row, row, q_out[:, :1], identity_rope(40, 64))
    assert math.isnan(float(cache.v_scales[at[1], 0, 0])) == (fmt == "int8")
    assert float(ref.values(cache.k_pages, cache.k_scales)[at[0], 0, 15, 0]) == 1.0
    cache.kv_len.zero_()
    h.append(cache, q[:, :1], row, row, q_out[:, :1], identity_rope(40, 64))
    assert (ref.values(cache.v_pages, cache.v_scales)[at, 0, 0] == 1).all()
    assert float(cache.v_scales[at[1], 0, 0]) == ref.scale_of(1.0, fmt)
    h.close()


def test_append_zeros_behind_rows_of_any_scale(pkg):
    for fmt in ref.MOST:
        h, cache, q, k, v, q_out, _ = append_case(pkg, D=64, dtype="f32", fmt=fmt, page=16, r=16, lens=[3, 3], counts=[4, 4], Hkv=1)
        for scale in (1e-40, 0.0, 2.0 ** -126, 0.3):
            cache.k_scales.fill_(scale)
            before = ref.codes_of(cache.k_pages)
            h.append(cache, q, torch.zeros_like(k), v, q_out, identity_rope(40, 64))
            now = ref.codes_of(cache.k_pages)
            p = cache.block_table.cpu()[:, 0].long()
            assert (now[p, 0, 3:7] == 0).all() and torch.equal(now[p, 0, :3], before[p, 0, :3])
            assert (cache.k_scales[p.cuda(), 0, 0] == scale).all()
        h.close()


def test_append_rows_without_a_place(pkg):
    for fmt in ref.MOST:
        h, cache, q, k, v, q_out, n_new = append_case(pkg, D=64, dtype="bf16", fmt=fmt, page=8, r=4, lens=[8, 8, 8, 8], counts=[9, 9, 9, 9], Hkv=1)
        rope, rows = identity_rope(60, 64), cache.rows
        before = [t.clone() for t in (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scales, cache.v_scales)]

        def same():
            now = (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scales, cache.v_scales)
            return all(torch.equal(a, b) for a, b in zip(before, now))

        for bad in (-3, -1, -2 ** 31, rows, rows + 1, 2 ** 31 - 1):
            cache.kv_len.fill_(bad)
            h.append(cache, q, k, v, q_out, rope, pos=torch.zeros_like(cache.kv_len), n_new=n_new)
            assert h.status() == 2 and same(), bad
        cache.kv_len.fill_(8)
        cache.block_table[:, 1:] = 2 ** 30
        h.append(cache, q, k, v, q_out, rope, n_new=n_new)
        assert h.status() == 16 and same()
        h.append(cache, q, k, v, q_out, rope, n_new=torch.full_like(n_new, 0))
        assert h.status() == 0 and same()
        h.close()
    # of rows that run over the table's end those before it are stored
    lens, fmt = [0], "int8"
    h, cache, q, k, v, q_out, n_new = append_case(pkg, D=64, dtype="bf16", fmt=fmt, page=8, r=4, lens=lens, counts=[20], Hkv=1)
    cache.kv_len.fill_(cache.rows - 5)
    want = stored(cache, "v", [cache.rows - 5], v, [5], fmt)
    h.append(cache, q, k, v, q_out, identity_rope(60, 64), pos=torch.zeros_like(cache.kv_len))
    assert h.status() == 2
    assert torch.equal(ref.codes_of(cache.v_pages), want[0]) and torch.equal(cache.v_scales.cpu().double(), want[1])
    h.close()


# -------------------------------------------------------------------- read

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Hkv,page,r,layout", [(2, 16, 16, "heads_first"), (8, 24, 6, "rows_first"), (3, 5, 1, "interleaved"), (1, 128, 64, "heads_first")])
def test_read(pkg, fmt, dtype, D, Hkv, page, r, layout):
    lens = [200, 17, 90]
    h, cache, *_ = setup(pkg, Hq=Hkv, Hkv=Hkv, D=D, dtype=dtype, fmt=fmt, page=page, r=r, lens=lens, layout=layout, wild=False)
    kv, vv, table = ref.values(cache.k_pages, cache.k_scales), ref.values(cache.v_pages, cache.v_scales), cache.block_table.cpu().long()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for n, start, count in ((90, i32(3, 0, 0), i32(90, 17, 33)), (16, None, None), (1, i32(199, 16, 5), None), (17, None, i32(0, 1, 17))):
        base = torch.full((3, Hkv, n + 2, D), 7.0, dtype=DT[dtype], device="cuda")
        k_out, v_out = base[:, :, :n].transpose(1, 2), torch.full((3, n, Hkv, D), 7.0, dtype=DT[dtype], device="cuda")
        h.read(cache, k_out, v_out, start=start, n_rows=count)
        assert h.status() == 0
        for b in range(3):
            m = n if count is None else int(count[b])
            slot = torch.arange(m) + (0 if start is None else int(start[b]))
            for out, vals in ((k_out, kv), (v_out, vv)):
                want = vals[table[b, slot // page], :, slot % page].float().to(DT[dtype])
                assert torch.equal(out[b, :m].cpu(), want) and (out[b, m:] == 7).all()
        assert (base[:, :, n:] == 7).all()
    h.close()


def test_read_outside_the_table(pkg):
    h, cache, *_ = setup(pkg, Hq=2, Hkv=2, D=64, dtype="bf16", fmt="int8", page=8, r=8, lens=[30, 30], room=0, wild=False)
    k_out, v_out = (torch.full((2, 9, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for first in (-3, 28, -2 ** 31, 2 ** 31 - 1):
        h.read(cache, k_out, v_out, start=torch.tensor([first, 0], dtype=torch.int32).cuda())
        assert h.status() == 2
        slot = first + torch.arange(9)
        inside = (slot >= 0) & (slot < cache.rows)
        assert (k_out[0][~inside.cuda()] == 0).all() and (v_out[0][~inside.cuda()] == 0).all()
        assert (k_out[0][inside.cuda()].abs().amax(-1) > 0).all()
    h.read(cache, k_out, v_out, n_rows=torch.tensor([-1, 10], dtype=torch.int32).cuda())
    assert h.status() == 4
    cache.block_table[1, 0] = cache.fields.n_pages
    h.read(cache, k_out, v_out)
    assert h.status() == 16 and (k_out[1, :8] == 0).all() and (k_out[1, 8].abs().amax(-1) > 0).all()
    h.close()


# --------------------------------------------------------------- together

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_decode_loop_as_a_graph(pkg, fmt):
    """Append and windowed attention, captured once, against the same calls by hand and
    the 64-bit form over what the cache then holds; then the rows read back."""
    B, Hq, Hkv, D, page, steps = 3, 8, 2, 128, 16, 40
    lens = [0, 13, 100]
    g = rng(4)
    outs = []
    for graph in (False, True):
        h, cache, *_ = setup(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype="bf16", fmt=fmt, page=page, r=16, lens=lens, room=4, wild=False)
        cache.k_scales.fill_(2.0 ** -12)
        cache.v_scales.fill_(2.0 ** -12)
        g.manual_seed(5)
        q, k, v = (torch.randn(steps, B, 1, H, D, generator=g).to(torch.bfloat16).cuda() for H in (Hq, Hkv, Hkv))
        q1, k1, v1, q_out = (torch.zeros_like(x[0]) for x in (q, k, v, q))
        out, rope = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device="cuda"), pkg.rope_table(300, D)
        gain = torch.ones(D, dtype=torch.bfloat16, device="cuda")

        def step():
            h.append(cache, q1, k1, v1, q_out, rope, g_q=gain, g_k=gain)
            h.attend(cache, q_out.view(B, Hq, D), out, window=32, sinks=4)
            cache.kv_len.add_(1)

        run = step
        if graph:
            state = [t.clone() for t in (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scales, cache.v_scales, cache.kv_len)]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                step()
            for t, s in zip((cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scales, cache.v_scales, cache.kv_len), state):
                t.copy_(s)
            run = cg.replay
        got = []
        for i in range(steps):
            q1.copy_(q[i]), k1.copy_(k[i]), v1.copy_(v[i])
            run()
            got.append(out.clone())
        assert h.status() == 0
        outs.append(torch.stack(got))
    assert torch.equal(outs[0], outs[1])
    now = [n + steps for n in lens]
    kv, vv = ref.values(cache.k_pages, cache.k_scales), ref.values(cache.v_pages, cache.v_scales)
    o, _, _, to, _, _ = ref.attend(q_out.view(B, Hq, D), kv, vv, cache.block_table, now, D ** -0.5, 32, 4, cache.v_scales.cpu())
    within(outs[1][-1].cpu(), o, to, "last step")
    k_rows, v_rows = (torch.zeros(B, max(now), Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    h.read(cache, k_rows, v_rows, n_rows=cache.kv_len)
    assert h.status() == 0
    # the values that were appended, within half a step of int8 (and of each growth before) or e4m3's 2^-4
    for b, n in enumerate(lens):
        x = v[:, b, 0].float().cpu()
        err = (v_rows[b, n:n + steps].float().cpu() - x).abs()
        assert (err <= (2.0 ** -4 * x.abs() + 2.0 ** -9 if fmt == "e4m3" else 4.5 / 127 * 2)).all()
    h.close()


def test_other_streams_and_two_handles(pkg):
    a = setup(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", fmt="e4m3", page=16, r=16, lens=[5000], wild=False)
    b = setup(pkg, Hq=8, Hkv=2, D=128, dtype="bf16", fmt="int8", page=16, r=16, lens=[7000], wild=False)
    want = []
    for h, cache, q, out, *_ in (a, b):
        h.attend(cache, q, out, added=0)
        want.append(out.clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for (h, cache, q, out, *_), s in zip((a, b), streams):
            with torch.cuda.stream(s):
                h.attend(cache, q, out, added=0)
    torch.cuda.synchronize()
    assert torch.equal(a[3], want[0]) and torch.equal(b[3], want[1])
    assert a[0].status() == 0 and b[0].status() == 0


def test_one_handle_serves_both_kinds_of_cache(pkg):
    h, codes, q, out, lse, scale, _ = setup(pkg, Hq=8, Hkv=2, D=64, dtype="f32", fmt="int8", page=16, r=16, lens=[300, 20], wild=False)
    k, v = (ref.values(p, s).float().cuda() for p, s in ((codes.k_pages, codes.k_scales), (codes.v_pages, codes.v_scales)))
    plain = h.cache(k, v, codes.block_table, codes.kv_len)
    h.attend(codes, q, out, added=0)
    again = torch.empty_like(out)
    h.attend(plain, q, again, added=0)
    o, _, _, to, _, _ = ref.attend(q, k.cpu().double(), v.cpu().double(), codes.block_table, [300, 20], scale, v_scales=codes.v_scales.cpu())
    within(out.cpu(), o, to + 2 * U * o.abs())
    within(again.cpu(), o, to)
    h.close()


def test_refusals(pkg):
    import ctypes
    h, cache, q, out, lse, _, _ = setup(pkg, Hq=8, Hkv=2, D=64, dtype="bf16", fmt="int8", page=16, r=16, lens=[30, 20], wild=False)
    lib, s = h.lib, cache.scales
    at = (q.data_ptr(), out.data_ptr(), None, None)

    def attend(scales, added=0, window=-1, sinks=0):
        return lib.prism_paged_attend_codes(h.h, cache.ref, None if scales is None else ctypes.byref(scales), added, window, sinks, *at)

    Scales = type(s)
    assert attend(s) == 0
    assert attend(None) == 1 and attend(Scales(None, s.v_scales, 1, 16)) == 1 and attend(Scales(s.k_scales, s.v_scales, 2, 16)) == 1
    assert attend(Scales(s.k_scales + 2, s.v_scales, 1, 16)) == 1 and b"aligned" in lib.prism_paged_error(h.h)
    for rows in (0, -1, 5, 32):
        assert attend(Scales(s.k_scales, s.v_scales, 1, rows)) == 2
        assert b"scale_rows" in lib.prism_paged_error(h.h)
    assert attend(s, added=-1) == 1 and attend(s, window=4, sinks=-1) == 1
    with pytest.raises(ValueError):
        h.attend(cache, q.float(), out)
    rows = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        h.read(cache, rows, rows[:, :2])
    with pytest.raises(pkg.PrismError):
        h.read(cache, rows[:, :1].expand(2, 3, 2, 64), rows)
    with pytest.raises(pkg.PrismError):
        h.read(cache, rows[:, :0], rows[:, :0])
    with pytest.raises(ValueError):
        h.read(cache, rows, rows, start=torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert h.status() == 0
    h.close()
