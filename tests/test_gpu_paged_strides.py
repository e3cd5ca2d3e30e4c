"""Strides of dimensions of one element: torch leaves them as it likes, and no call uses them."""
from __future__ import annotations

import pytest
import torch

from .test_gpu_paged import DT, handle, pkg  # noqa: F401

pytestmark = pytest.mark.gpu


def odd(t, dim, stride):
    """The same values with another stride along a dimension of one element."""
    assert t.shape[dim] == 1
    s = list(t.stride())
    s[dim] = stride
    return t.as_strided(t.shape, s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,dim", [(1, 3, 4, 0), (3, 1, 4, 1), (3, 3, 1, 2)])
def test_rows_of_one_batch_row_or_head(pkg, dtype, B, n, H, dim):  # noqa: F811
    g, dt, D = torch.Generator(device="cuda").manual_seed(1), DT[dtype], 64
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    q, k, v, dq, dk = (rand(B, n, H, D) for _ in range(5))
    gains, rope = [rand(D) for _ in range(2)], pkg.rope_table(16, D)
    pos = torch.arange(B, dtype=torch.int32, device="cuda")
    h = handle(pkg, H, H, D, dtype, max_batch=B, max_pages=1)
    got = []
    for f in (lambda t: t, lambda t: odd(t, dim, 5), lambda t: odd(t, dim, 0)):
        o = [torch.zeros(B, n, H, D, dtype=dt, device="cuda") for _ in range(5)]
        dg = torch.zeros(2, D, device="cuda")
        pages = [torch.zeros(B, H, 16, D, dtype=dt, device="cuda") for _ in range(2)]
        cache = h.cache(*pages, pos.view(B, 1), pos)
        h.qk_norm_rope(f(q), f(k), f(o[0]), f(o[1]), rope, pos, g_q=gains[0], g_k=gains[1])
        h.qk_norm_rope_backward(f(dq), f(dk), f(q), f(k), f(o[2]), f(o[3]), rope, pos, g_q=gains[0], g_k=gains[1], dg_q=dg[0], dg_k=dg[1])
        h.append(cache, f(q), f(k), f(v), f(o[4]), rope, g_q=gains[0], g_k=gains[1])
        assert h.status() == 0
        got.append([*o, dg, *pages])
    for a in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(a, got[0]))
    h.close()


@pytest.mark.parametrize("n_pages,H,page,dim", [(1, 2, 16, 0), (3, 1, 16, 1), (5, 2, 1, 2)])
def test_pages_of_one_page_head_or_row(pkg, n_pages, H, page, dim):  # noqa: F811
    """K and V with another such stride each."""
    g, D = torch.Generator(device="cuda").manual_seed(2), 64
    k, v = (torch.randn(n_pages, H, page, D, generator=g, device="cuda") for _ in range(2))
    w = torch.rand(n_pages, H, page, generator=g, device="cuda")
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda").view(1, -1)
    L = torch.tensor([min(n_pages * page - 2, 30)], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 2 * H, D, generator=g, device="cuda")
    h = handle(pkg, 2 * H, H, D, "f32", page_size=page, max_pages=n_pages, track_weights=True)
    got = []
    for f in (lambda t, s: t, lambda t, s: odd(t, dim, s), lambda t, s: odd(t, dim, 0)):
        wt, out = w.clone(), torch.empty_like(q)
        h.attend(h.cache(f(k, 3), f(v, 7), table, L, weights=wt), q, out, added=0)
        assert h.status() == 0
        got.append((out, wt))
    for a in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(a, got[0]))
    h.close()
