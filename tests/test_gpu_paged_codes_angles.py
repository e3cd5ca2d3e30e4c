"""Keys normed and rotated by real angles as they are quantised: every form that the
rows of a block take (several short blocks to a warp, one, two and four warps, rows read
again, angles beyond those that are kept, tiles one after the other), each code held to
the interval that fp32 arithmetic leaves it."""
from __future__ import annotations

import pytest
import torch

from . import codes_check as check
from . import codes_ref as ref
from . import paged_ref
from .test_gpu_paged_codes import DT, EPS, code_pool, rng, tables

pytestmark = pytest.mark.gpu


def append_and_check(*, dtype, D, fmt, Hkv, page, r, lens, counts, gains, Hq=4, seed=0, theta=10000.0, layout="heads_first"):
    import paper_2602_01762_gb300 as p
    g = rng(seed)
    B, n = len(lens), max(max(counts), 1)
    pages = -(-(max(lens) + n) // page) + 1
    n_pages, table = tables(g, B, pages)
    k_pages, v_pages, ks, vs = code_pool(g, n_pages, Hkv, page, D, fmt, r, layout)
    # as an append leaves them, from far below the new rows to far above
    ks, vs = (torch.exp2(torch.floor(torch.log2(s)) + torch.randint(-6, 2, s.shape, generator=g).cuda()) for s in (ks, vs))
    q, k, v = (torch.randn(B, n, H, D, generator=g) for H in (Hq, Hkv, Hkv))
    size = check.interleaved_sizes(g, B, n, Hkv, r)
    q, k, v = (x.to(DT[dtype]).cuda() for x in (q, k * size, v * size.roll(1, 1)))
    g_q, g_k = ((torch.randn(D, generator=g) * 0.3 + 1).to(DT[dtype]).cuda() for _ in range(2)) if gains else (None, None)
    pos = [int(x) for x in torch.randint(0, 400, (B,), generator=g)]
    rope = p.rope_table(400 + n, D, theta)
    h = p.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=B, max_pages=pages, rms_eps=EPS)
    cache = h.cache(k_pages, v_pages, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), k_scales=ks, v_scales=vs)
    q_out = torch.zeros_like(q)

    def state(name):
        return ref.codes_of(getattr(cache, name + "_pages")), getattr(cache, name + "_scales").cpu().double()

    before = {name: state(name) for name in "kv"}
    h.append(cache, q, k, v, q_out, rope, g_q=g_q, g_k=g_k, pos=torch.tensor(pos, dtype=torch.int32).cuda(),
             n_new=torch.tensor(counts, dtype=torch.int32).cuda())
    assert h.status() == 0
    rows = {"k": [check.keys(k[b, :c], g_k, rope, pos[b], EPS) for b, c in enumerate(counts)],
            "v": [(v[b, :c].cpu().double(), torch.zeros(c, Hkv, D, dtype=torch.float64)) for b, c in enumerate(counts)]}
    for name in "kv":
        check.check_stored(before[name], state(name), table, lens, rows[name], counts, fmt, name)
    for b, c in enumerate(counts):
        want, tol = paged_ref.norm_rope(q[b, :c], g_q, rope, pos[b], EPS)
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        paged_ref.within(q_out[b, :c], want, tol + half * want.abs(), "q")
        assert (q_out[b, c:] == 0).all()
    h.close()


# blocks of a quarter of a warp's rows to beyond what four warps keep, in multiples of each form's rows and not
BLOCKS = [(8, 1), (16, 2), (12, 3), (16, 4), (24, 6), (8, 8), (24, 12), (16, 16), (48, 24), (32, 32), (64, 64), (100, 100), (128, 128), (200, 200)]


@pytest.mark.parametrize("gains", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page,r", BLOCKS)
def test_rows_of_every_block_size(dtype, D, page, r, gains):
    append_and_check(dtype=dtype, D=D, fmt="e4m3" if gains else "int8", Hkv=3, Hq=6, page=page, r=r, lens=[0, 1, r - 1, r // 2 + 1, 2 * r, 77],
                     counts=[3 * r + 1, 2, 1, 230, 0, 5], gains=gains, seed=r)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page,r", [(16, 16), (24, 24), (64, 64), (100, 100), (128, 128)])
def test_one_token_behind_any_row(fmt, dtype, D, page, r):
    lens = list(range(0, 2 * r, max(r // 17, 1)))
    append_and_check(dtype=dtype, D=D, fmt=fmt, Hkv=2, page=page, r=r, lens=lens, counts=[int(b % 7 > 0) for b in range(len(lens))], gains=r % 3 > 0, seed=r)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("page,r", [(16, 16), (32, 32), (64, 64)])
def test_a_few_rows_to_verify(fmt, dtype, D, page, r):
    """2 to 16 rows behind any number of rows, as a draft's rows are stored before they are verified."""
    lens = list(range(0, 2 * r, max(r // 11, 1)))
    append_and_check(dtype=dtype, D=D, fmt=fmt, Hkv=8, Hq=8, page=page, r=r, lens=lens, counts=[2 + b * 5 % 15 for b in range(len(lens))], gains=True, seed=r)


def chained(r, dtype, D, turns):
    """New rows of each of four sequences that give a CTA `turns` tiles."""
    warp_rows = 32 // (D // 2 // (8 if dtype == "bf16" else 4))
    per = warp_rows // r if r < warp_rows and warp_rows % r == 0 else 1
    ctas = 5 if r <= warp_rows else 4 if r <= 2 * warp_rows else 3           # an SM's
    tiles = turns * ctas * torch.cuda.get_device_properties(0).multi_processor_count
    return (tiles // 4 + 2) * r * per


@pytest.mark.parametrize("turns", [2, 3, 4])
@pytest.mark.parametrize("dtype,D,Hkv,r", [("bf16", 128, 1, 1), ("bf16", 128, 2, 2), ("bf16", 128, 1, 3), ("bf16", 128, 5, 4), ("bf16", 128, 1, 8),
                                           ("bf16", 128, 1, 16), ("bf16", 64, 3, 2), ("bf16", 64, 1, 8), ("bf16", 64, 1, 32), ("f32", 128, 1, 2),
                                           ("f32", 128, 1, 4), ("f32", 128, 2, 8), ("f32", 128, 2, 16), ("f32", 64, 1, 4), ("f32", 64, 2, 32)])
def test_tiles_one_after_the_other(dtype, D, Hkv, r, turns):
    n = chained(r, dtype, D, turns)
    append_and_check(dtype=dtype, D=D, fmt="int8" if turns == 3 else "e4m3", Hkv=Hkv, Hq=Hkv, page=max(16 // r, 1) * r, r=r, lens=[0, r // 2, 5, 3 * r - 1],
                     counts=[n, n - r - 1, n // 2, n - 3 * r], gains=turns == 2, seed=r + turns)


@pytest.mark.parametrize("layout", ["rows_first", "interleaved"])
def test_other_layouts(layout):
    for fmt in ref.MOST:
        append_and_check(dtype="bf16", D=128, fmt=fmt, Hkv=4, Hq=8, page=16, r=8, lens=[3, 16, 40], counts=[33, 8, 20], gains=True, layout=layout)
