"""Paged-cache operators without a GPU: what the C entry points answer before they
touch a device, and the 64-bit forms the GPU tests compare with."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

from . import paged_ref as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2602_01762_gb300 import build, library
    build.build()
    return library()


def test_null_handles_are_refused(lib):
    assert lib.prism_qk_norm_rope(None, None, None) == 1
    assert lib.prism_qk_norm_rope_backward(None, None, None, None) == 1
    assert lib.prism_paged_append(None, None, None, None) == 1
    assert lib.prism_paged_attend(None, None, 1, None, None, None, None) == 1
    assert lib.prism_paged_evict(None, None, None, 1, 0, 0, None, None) == 1
    assert lib.prism_paged_status(None, None, None) == 1
    assert lib.prism_paged_destroy(None) == 0
    assert b"null" in lib.prism_paged_error(None)


@pytest.mark.parametrize("field,value", [("head_dim", 80), ("n_kv_heads", 3), ("n_kv_heads", 0), ("page_size", 0), ("max_batch", 0),
                                         ("max_pages", 0), ("dtype", 7), ("rms_eps", -1.0), ("softmax_scale", float("nan")),
                                         ("max_pages", 2 ** 27), ("max_batch", 2 ** 24)])
def test_create_refuses_before_touching_cuda(lib, field, value):
    from paper_2602_01762_gb300.paged import _PagedConfig
    cfg = _PagedConfig(8, 2, 64, 1, 16, 4, 64, 0, 0.0, 1e-5)
    setattr(cfg, field, value)
    out = ctypes.c_void_p()
    assert lib.prism_paged_create(ctypes.byref(cfg), 0, ctypes.byref(out)) in (1, 3)
    assert not out.value
    assert lib.prism_paged_create(None, 0, ctypes.byref(out)) == 1


def test_rope_table_is_the_rotation():
    from paper_2602_01762_gb300 import rope_table
    t = rope_table(50, 64, 10000.0, device="cpu")
    assert t.shape == (50, 2, 32) and t.dtype == torch.float32
    assert torch.equal(t[0, 0], torch.ones(32)) and torch.equal(t[0, 1], torch.zeros(32))
    want = 37 * 10000.0 ** (-2 * 5 / 64)
    assert abs(float(t[37, 0, 5]) - np.cos(want)) < 1e-7 and abs(float(t[37, 1, 5]) - np.sin(want)) < 1e-7


def test_reference_scores_depend_on_distance_alone():
    g = torch.Generator().manual_seed(1)
    from paper_2602_01762_gb300 import rope_table
    t = rope_table(90, 64, 10000.0, device="cpu")
    q, k = torch.randn(1, 1, 64, generator=g), torch.randn(1, 1, 64, generator=g)
    dots = [float((ref.norm_rope(q, None, t, p + 13, 0.0)[0] * ref.norm_rope(k, None, t, p, 0.0)[0]).sum()) for p in (0, 5, 60)]
    assert max(dots) - min(dots) < 1e-5
    y, _ = ref.norm_rope(q, torch.ones(64), t, 7, 0.0)
    assert abs(float((y * y).mean()) - 1) < 1e-6


def test_reference_gradient_against_differences():
    g = torch.Generator().manual_seed(2)
    from paper_2602_01762_gb300 import rope_table
    t = rope_table(20, 64, 10000.0, device="cpu")
    x, dy = (torch.randn(3, 2, 64, generator=g).double() for _ in range(2))
    gain = torch.randn(64, generator=g).double()
    dx, dg, _, _ = ref.norm_rope_grad(x, gain, dy, t, 4, 1e-5)

    def total(x, gain):
        return float((ref.norm_rope(x, gain, t, 4, 1e-5)[0] * dy).sum())

    u, w, step = torch.randn(x.shape, generator=g).double(), torch.randn(64, generator=g).double(), 1e-5
    assert abs((total(x + step * u, gain) - total(x - step * u, gain)) / (2 * step) - float((dx * u).sum())) < 1e-6
    assert abs((total(x, gain + step * w) - total(x, gain - step * w)) / (2 * step) - float((dg * w).sum())) < 1e-6


def test_reference_attention_of_equal_keys_is_the_mean():
    g = torch.Generator().manual_seed(3)
    k = torch.ones(4, 1, 8, 64)
    v = torch.randn(4, 1, 8, 64, generator=g)
    table = torch.tensor([[2, 0]])
    q = torch.randn(1, 2, 64, generator=g)
    out, lse, w, *_ = ref.attend(q, k, v, table, [13], 0.125)
    mean = torch.cat([v[2, 0], v[0, 0, :5]]).double().mean(0)
    assert (out[0] - mean).abs().max() < 1e-12
    assert torch.allclose(w[0], torch.full((1, 13), 2 / 13, dtype=torch.float64))
    assert torch.allclose(lse[0], np.log(13) + q[0].double().sum(1) * 0.125)
    out, lse, w, *_ = ref.attend(q, k, v, table, [0], 0.125)
    assert (out == 0).all() and (lse == -float("inf")).all()


def test_reference_eviction_order():
    w = np.array([9, 1, float("nan"), 5, 5, -0.0, 0.0, 7, 2, 3], np.float32)
    assert ref.kept_rows(w, 10, 5, 1, 1).tolist() == [0, 3, 4, 7, 9]
    assert ref.kept_rows(w, 10, 8, 0, 0).tolist() == [0, 1, 3, 4, 5, 7, 8, 9]
    assert ref.kept_rows(w, 3, 5, 1, 1).tolist() == [0, 1, 2]
