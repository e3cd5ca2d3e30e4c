"""The cache held in 8 bits without a GPU: the 64-bit forms, and what the binding and
the C entry points refuse before they touch a device."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from . import codes_ref as ref


@pytest.fixture(scope="module")
def pkg():
    from paper_2602_01762_gb300 import build
    build.build()
    import paper_2602_01762_gb300 as p
    p.library()
    return p


def host_handle(pkg, Hq=4, Hkv=2, D=64, page=16):
    """The binding's checks alone: a handle without a device."""
    h = pkg.PagedAttention.__new__(pkg.PagedAttention)
    h.h, h.lib, h.tdtype, h.device, h._index, h._dims = None, pkg.library(), torch.bfloat16, torch.device("cpu"), -1, (D,)
    h.n_q_heads, h.n_kv_heads, h.head_dim, h.page_size = Hq, Hkv, D, page
    h._key = (h.tdtype, h.device, (Hkv, page, D))
    return h


def host_cache(h, n=3, blocks=4, dtype=torch.int8, **kw):
    k = torch.zeros(n, h.n_kv_heads, h.page_size, h.head_dim, dtype=dtype)
    a = dict(k_pages=k, v_pages=k.clone(), block_table=torch.zeros(1, 2, dtype=torch.int32), kv_len=torch.zeros(1, dtype=torch.int32),
             k_scales=torch.ones(n, h.n_kv_heads, blocks), v_scales=torch.ones(n, h.n_kv_heads, blocks))
    a.update(kw)
    return h.cache(**a)


def test_nearest_is_torch_s_rounding_where_it_has_one():
    g = torch.Generator().manual_seed(0)
    y = torch.cat([torch.randn(20000, generator=g) * 10.0 ** (torch.rand(20000, generator=g) * 5 - 4),
                   torch.arange(-4480, 4481) / 10.0, torch.arange(-2 ** 7, 2 ** 7) * 2.0 ** -11]).clamp(-448, 448)
    assert torch.equal(ref.nearest(y.double(), "e4m3"), y.to(torch.float8_e4m3fn).to(torch.float32).double())
    half = torch.arange(-127, 127) + 0.5
    assert torch.equal(ref.nearest(half.double(), "int8"), torch.tensor(np.rint(half.numpy()), dtype=torch.float64))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scale_is_the_smallest_power_that_holds(fmt):
    for top in (448.0, 448.1, 127.0, 126.9, 127.1, 3.5, 3.96875, 3.97, 1e-30, 3e38, 2.0 ** -140):
        s = ref.scale_of(top, fmt)
        assert top <= ref.MOST[fmt] * s and np.log2(s) % 1 == 0
        assert s == 2.0 ** -126 or top > ref.MOST[fmt] * s / 2
    assert ref.scale_of(0.0, fmt) == 0.0 and ref.scale_of(448.0, "e4m3") == 1.0 and ref.scale_of(127.0, "int8") == 1.0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_stored_rows_are_within_a_step(fmt):
    """Rows stored one by one in a block that grows: half a step of the block's own
    rounding and, for int8, half a step of every growth before."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(1, 16, 1, 64, generator=g, dtype=torch.float64) * torch.logspace(-3, 1, 16, dtype=torch.float64)[None, :, None, None]
    codes, scales = torch.zeros(1, 1, 16, 64, dtype=torch.float64), torch.full((1, 1, 1), 9.0, dtype=torch.float64)
    table = torch.zeros(1, 1, dtype=torch.int32)
    for i in range(16):
        ref.store(codes, scales, table, [i], x[:, i:i + 1], [1], fmt)
    s = float(scales)
    assert s == ref.scale_of(float(x.abs().max()), fmt)
    err = (codes[0, 0] * s - x[0, :, 0]).abs()
    # e4m3: 2^-4 of the value, or steps of 2^-9 s (each growth adds half a step of its own scale)
    bound = s * torch.ones_like(err) if fmt == "int8" else 2.0 ** -4 * x[0, :, 0].abs() + 2.0 ** -9 * s
    assert (err <= bound).all()


def test_seen_rows():
    assert ref.seen(10, None, 3).tolist() == list(range(10))
    assert ref.seen(10, 4, 2).tolist() == [0, 1, 6, 7, 8, 9]
    assert ref.seen(10, 9, 5).tolist() == list(range(10))
    assert ref.seen(10, 0, 0).tolist() == [] and ref.seen(0, 5, 5).tolist() == []


def test_attention_of_all_rows_is_the_plain_one():
    from . import paged_ref
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(5, 2, 8, 64, generator=g, dtype=torch.float64) for _ in range(2))
    q, table = torch.randn(2, 4, 64, generator=g), torch.tensor([[4, 0, 2], [1, 3, 0]], dtype=torch.int32)
    want, got = paged_ref.attend(q, k, v, table, [19, 3], 0.125), ref.attend(q, k, v, table, [19, 3], 0.125)
    assert all(torch.allclose(a, b, rtol=1e-12, atol=0) for a, b in zip(want[:2], got[:2]))
    few = ref.attend(q, k, v, table, [19, 3], 0.125, window=19)
    assert torch.equal(few[0], got[0])


def test_null_arguments_are_refused(pkg):
    lib = pkg.library()
    assert lib.prism_paged_attend_window(None, None, 1, 4, 0, None, None, None, None) == 1
    assert lib.prism_paged_attend_codes(None, None, None, 1, -1, 0, None, None, None, None) == 1
    assert lib.prism_paged_append_codes(None, None, None, None, None) == 1
    assert lib.prism_paged_read_codes(None, None, None, None, None, 1, None, None, None) == 1
    assert b"null" in lib.prism_paged_error(None)


def test_the_binding_refuses(pkg):
    h = host_handle(pkg)
    cache = host_cache(h)
    assert cache.scales.scale_rows == 4 and cache.scales.format == 1
    assert host_cache(h, blocks=16, dtype=torch.float8_e4m3fn).scales.scale_rows == 1
    ones = torch.ones(3, 2, 4)
    for bad in (dict(k_scales=None), dict(v_scales=None), dict(v_scales=torch.ones(3, 2, 8)), dict(k_scales=torch.ones(3, 2, 5), v_scales=torch.ones(3, 2, 5)),
                dict(k_scales=ones.double(), v_scales=ones.double()), dict(k_scales=torch.ones(3, 2), v_scales=torch.ones(3, 2)),
                dict(k_scales=torch.ones(3, 2, 0), v_scales=torch.ones(3, 2, 0)), dict(k_scales=torch.ones(3, 2, 32), v_scales=torch.ones(3, 2, 32)),
                dict(v_pages=torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn)), dict(weights=torch.zeros(3, 2, 16)),
                dict(v_scales=torch.ones(3, 4, 2).transpose(1, 2))):
        with pytest.raises(ValueError):
            host_cache(h, **bad)
    for dtype in (torch.bfloat16, torch.uint8, torch.float8_e5m2):
        with pytest.raises(ValueError):
            host_cache(h, dtype=dtype)
    plain = host_cache(h, dtype=torch.bfloat16, k_scales=None, v_scales=None)
    q, out = torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    rows = torch.zeros(1, 5, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="window"):
        h.attend(cache, q, out, window=-1)
    with pytest.raises(ValueError, match="sinks"):
        h.attend(plain, q, out, sinks=4)
    with pytest.raises(ValueError, match="8 bits"):
        h.read(plain, rows, rows.clone())
    for src, dst in ((cache, plain), (plain, cache)):
        with pytest.raises(ValueError, match="8 bits"):
            h.evict(src, dst, torch.zeros(1, 2, 8, dtype=torch.int32))
    with pytest.raises(TypeError):
        h.attend(None, q, out, window=3)
