"""Operators over a paged key-value cache (the paged section of
``include/prism.h``): the per-head norm of queries and keys with the position
rotation, stored into the cache (:meth:`PagedAttention.append`) or dense with
its gradient (:meth:`PagedAttention.qk_norm_rope`,
:meth:`PagedAttention.qk_norm_rope_backward`), the attention of one new token
(:meth:`PagedAttention.attend`), to every row or to a sliding window, eviction by
accumulated attention weight (:meth:`PagedAttention.evict`), and rows of a cache held
in 8 bits read back (:meth:`PagedAttention.read`).

A decode step of one layer::

    att = PagedAttention(n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16,
                         max_batch=B, max_pages=P, track_weights=True)
    cache = att.cache(k_pages, v_pages, block_table, kv_len, weights=weights)
    rope = rope_table(max_positions, 128, theta=500000.0)

    att.append(cache, q, k, v, q_out, rope, g_q=g_q, g_k=g_k, pos=pos)   # row kv_len[b]
    att.attend(cache, q_out.view(B, 32, 128), out)                       # over kv_len[b] + 1 rows
    kv_len += 1; pos += 1

and, when the cache has grown past its budget,
``att.evict(cache, other_cache, kept, sinks=4, recent=512)``.  Attention to the last
rows and a few first ones alone is ``att.attend(..., window=1024, sinks=4)``.

A cache held in 8 bits has pages of ``torch.float8_e4m3fn`` or ``torch.int8`` codes
and a scale for each block of rows, ``att.cache(k_pages, v_pages, block_table, kv_len,
k_scales=ks, v_scales=vs)``; ``append`` quantises into it, ``attend`` reads it as it is,
``read`` gives rows back in the handle's type.

As in the rest of the package the binding only checks and marshals: every
result is computed by the library's kernels on the current CUDA stream, and a
missing library raises.  Autograd records none of them: outputs carry no history,
also of inputs that require a gradient, and the norm's gradient is the call named
above.  Tensors belong to the caller; a call that uses a tensor
on another stream than the one it was allocated on needs the caller's
``record_stream``, as with any asynchronous torch operation.
"""
from __future__ import annotations

import ctypes
import struct

import torch

__all__ = ["PagedAttention", "PagedCache", "rope_table"]

_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class _PagedConfig(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "dtype", "page_size", "max_batch",
                                    "max_pages", "track_weights")] + [("softmax_scale", ctypes.c_float),
                                                                      ("rms_eps", ctypes.c_float)]


class _Cache(ctypes.Structure):
    _fields_ = [("k_pages", _vp), ("v_pages", _vp), ("page_stride", _i64), ("head_stride", _i64), ("row_stride", _i64),
                ("weights", _vp), ("block_table", _vp), ("kv_len", _vp), ("n_pages", _i32), ("table_pages", _i32),
                ("batch", _i32)]


class _Scales(ctypes.Structure):
    _fields_ = [("k_scales", _vp), ("v_scales", _vp), ("format", _i32), ("scale_rows", _i32)]


_CODES = {torch.float8_e4m3fn: 0, torch.int8: 1}

# prism_rows (five strided tensors of four words, five addresses, three sizes) and
# prism_row_grads (four strided tensors, two addresses)
_ROWS, _GRADS = struct.Struct("=20q5Q3i4x"), struct.Struct("=16q2Q")
_HEADS2 = struct.Struct("=8q")       # two prism_heads
_NONE = (0, 0, 0, 0)


def bind(lib: ctypes.CDLL) -> None:
    """Argument and result types of the paged entry points."""
    P = ctypes.POINTER
    C = P(_Cache)
    lib.prism_paged_create.argtypes = [P(_PagedConfig), _i32, P(_vp)]
    lib.prism_paged_destroy.argtypes = [_vp]
    lib.prism_qk_norm_rope.argtypes = [_vp, _vp, _vp]
    lib.prism_qk_norm_rope_backward.argtypes = [_vp, _vp, _vp, _vp]
    lib.prism_paged_append.argtypes = [_vp, C, _vp, _vp]
    lib.prism_paged_attend.argtypes = [_vp, C, _i32, _vp, _vp, _vp, _vp]
    lib.prism_paged_evict.argtypes = [_vp, C, C, _i32, _i32, _i32, _vp, _vp]
    S = P(_Scales)
    lib.prism_paged_attend_window.argtypes = [_vp, C, _i32, _i32, _i32, _vp, _vp, _vp, _vp]
    lib.prism_paged_append_codes.argtypes = [_vp, C, S, _vp, _vp]
    lib.prism_paged_read_codes.argtypes = [_vp, C, S, _vp, _vp, _i32, _vp, _vp, _vp]
    lib.prism_paged_attend_codes.argtypes = [_vp, C, S, _i32, _i32, _i32, _vp, _vp, _vp, _vp]
    lib.prism_paged_status.argtypes = [_vp, _vp, P(_i32)]
    lib.prism_paged_error.argtypes = [_vp]
    lib.prism_paged_error.restype = ctypes.c_char_p
    for f in ("prism_paged_create", "prism_paged_destroy", "prism_qk_norm_rope", "prism_qk_norm_rope_backward",
              "prism_paged_append", "prism_paged_attend", "prism_paged_evict", "prism_paged_status", "prism_paged_attend_window",
              "prism_paged_append_codes", "prism_paged_read_codes", "prism_paged_attend_codes"):
        getattr(lib, f).restype = ctypes.c_int


def rope_table(positions: int, head_dim: int, theta: float = 10000.0, device=0) -> torch.Tensor:
    """fp32 [positions, 2, head_dim / 2]: cosines and sines of
    position * theta^(-2j / head_dim), computed in fp64."""
    a = torch.arange(positions, dtype=torch.float64)[:, None] * (
        float(theta) ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim))
    return torch.stack([torch.cos(a), torch.sin(a)], 1).float().to(device)


class PagedCache:
    """A paged cache bound by :meth:`PagedAttention.cache`: its tensors, checked
    once, and the structs the calls pass on (``scales`` None: a cache of the handle's
    own type)."""

    def __init__(self, fields, tensors, batch, rows, dtype, device, heads, scales=None, k_scales=None, v_scales=None):
        self.fields, self.ref = fields, ctypes.byref(fields)
        self.scales, self.k_scales, self.v_scales = scales, k_scales, v_scales
        self.scales_ref = None if scales is None else ctypes.byref(scales)
        self.k_pages, self.v_pages, self.block_table, self.kv_len, self.weights = tensors
        self.batch, self.rows = batch, rows          # sequences; rows a block-table line holds
        self.key = (dtype, device, heads)


class PagedAttention:
    """Paged-cache operators of one attention layout on one GPU.

    ``dtype`` "bf16" or "f32" is that of queries, keys, values, gains and cache (but
    for one held in 8 bits);
    ``max_batch`` and ``max_pages`` bound the calls that take a cache;
    ``track_weights`` allots the workspace that accumulating attention weights
    needs; ``softmax_scale`` None means ``head_dim ** -0.5``.  A handle's calls
    share its workspace: keep them on one stream."""

    def __init__(self, *, n_q_heads, n_kv_heads, head_dim, page_size, max_batch, max_pages, dtype="bf16",
                 track_weights=False, softmax_scale=None, rms_eps=1e-5, device=0):
        from . import library
        if dtype not in ("bf16", "f32"):
            raise ValueError("dtype must be 'bf16' or 'f32'")
        self.h = None
        self.lib = library()
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device = torch.device("cuda", device)
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_size = n_q_heads, n_kv_heads, head_dim, page_size
        self.max_batch, self.max_pages, self.track_weights = max_batch, max_pages, bool(track_weights)
        cfg = _PagedConfig(n_q_heads, n_kv_heads, head_dim, 1 if dtype == "bf16" else 0, page_size, max_batch, max_pages,
                           int(bool(track_weights)), 0.0 if softmax_scale is None else float(softmax_scale), float(rms_eps))
        h = _vp()
        self._check(self.lib.prism_paged_create(ctypes.byref(cfg), device, ctypes.byref(h)))
        self.h = h
        self._index, self._dims = self.device.index, (head_dim,)
        self._rows, self._grads = ctypes.create_string_buffer(_ROWS.size), ctypes.create_string_buffer(_GRADS.size)
        self._kv_rows = ctypes.create_string_buffer(_HEADS2.size)
        self._k_rows_at = ctypes.addressof(self._kv_rows)
        self._v_rows_at = self._k_rows_at + _HEADS2.size // 2
        self._rows_at, self._grads_at = ctypes.addressof(self._rows), ctypes.addressof(self._grads)
        self._key = (self.tdtype, self.device, (n_kv_heads, page_size, head_dim))

    # ------------------------------------------------------------ checks
    def _check(self, status):
        if status:
            from . import PrismError
            raise PrismError(status, (self.lib.prism_paged_error(self.h) or b"").decode())

    def _refuse(self, t, what, name):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name}: expected a torch.Tensor")
        raise ValueError(f"{name}: expected {what} on {self.device}, got {t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")

    def _tensor(self, t, shape, dtype, name):
        """Address of a dense tensor of this device, shape and type."""
        try:
            if t.shape == shape and t.dtype is dtype and t.get_device() == self._index and t.is_contiguous():
                return t.data_ptr()
        except AttributeError:
            pass
        self._refuse(t, f"contiguous {dtype} {tuple(shape)}", name)

    def _heads(self, t, shape, name):
        """Address and strides of a [batch, rows, heads, D] tensor, D dense."""
        try:
            if t.shape == shape and t.dtype is self.tdtype and t.get_device() == self._index:
                b, r, h, d = t.stride()
                if d == 1:
                    return t.data_ptr(), b, r, h
        except AttributeError:
            pass
        self._refuse(t, f"{self.tdtype} {shape} with a dense head dimension", name)

    def _pack(self, shape_q, shape_k, q, k, v, q_out, k_out, rope, pos, g_q, g_k, n_new):
        """Checks a block of rows and writes its prism_rows."""
        heads, tensor, i32, B = self._heads, self._tensor, torch.int32, shape_q[0:1]
        n = rope.shape[0]
        _ROWS.pack_into(
            self._rows, 0, *heads(q, shape_q, "q"), *heads(k, shape_k, "k"), *(_NONE if v is None else heads(v, shape_k, "v")),
            *(_NONE if q_out is None else heads(q_out, shape_q, "q_out")), *(_NONE if k_out is None else heads(k_out, shape_k, "k_out")),
            0 if g_q is None else tensor(g_q, self._dims, self.tdtype, "g_q"),
            0 if g_k is None else tensor(g_k, self._dims, self.tdtype, "g_k"),
            tensor(rope, (n, 2, self.head_dim // 2), torch.float32, "rope"),
            0 if pos is None else tensor(pos, B, i32, "pos"), 0 if n_new is None else tensor(n_new, B, i32, "n_new"), n, B[0], shape_q[1])

    def _stream(self, stream):
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def _bound(self, cache):
        if not isinstance(cache, PagedCache):
            raise TypeError("expected a PagedCache (PagedAttention.cache)")
        if cache.key != self._key:
            raise ValueError("the cache was bound for another layout, type or device")
        return cache.ref

    # ------------------------------------------------------------ calls
    def cache(self, k_pages, v_pages, block_table, kv_len, weights=None, k_scales=None, v_scales=None) -> PagedCache:
        """Bind a paged cache.  ``k_pages``, ``v_pages`` [n_pages, Hkv, page_size,
        D], dense in D, with the same strides otherwise (a permuted view of [n_pages,
        page_size, Hkv, D] storage will do; dimensions of one element do not count);
        ``block_table`` int32 [batch, pages]; ``kv_len`` int32 [batch]; ``weights``
        fp32 [n_pages, Hkv, page_size].

        With ``k_scales`` and ``v_scales``, fp32 [n_pages, Hkv, page_size / r], a cache
        held in 8 bits: pages of ``torch.float8_e4m3fn`` or ``torch.int8``, a scale for
        each r rows of a page and head (``prism_paged_scales``), no weights."""
        n_pages = k_pages.shape[0]
        scales, dtype = None, self.tdtype
        if (k_scales is None) != (v_scales is None):
            raise ValueError("k_scales and v_scales are given together or not at all")
        if k_scales is not None:
            dtype = k_pages.dtype
            if dtype not in _CODES:
                raise ValueError(f"k_pages: expected torch.float8_e4m3fn or torch.int8 with scales, got {dtype}")
            if weights is not None:
                raise ValueError("a cache held in 8 bits has no weights")
            if k_scales.dim() != 3 or k_scales.shape[2] < 1 or self.page_size % k_scales.shape[2]:
                raise ValueError(f"k_scales: expected [n_pages, n_kv_heads, blocks], blocks a divisor of {self.page_size}")
            blocks = (n_pages, self.n_kv_heads, k_scales.shape[2])
            scales = _Scales(self._tensor(k_scales, blocks, torch.float32, "k_scales"), self._tensor(v_scales, blocks, torch.float32, "v_scales"),
                             _CODES[dtype], self.page_size // blocks[2])
        shape = (n_pages, self.n_kv_heads, self.page_size, self.head_dim)
        for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
            if t.dtype is not dtype or t.shape != shape or t.device != self.device:
                raise ValueError(f"{name}: expected {dtype} {shape} on {self.device}, got {t.dtype} {tuple(t.shape)} "
                                 f"on {t.device}")
            if t.stride(3) != 1 or any(a != b for n, a, b in zip(shape, t.stride(), k_pages.stride()) if n > 1):
                raise ValueError(f"{name}: K and V need the same strides and a dense head dimension")
        if block_table.dim() != 2:
            raise ValueError("block_table: expected two dimensions")
        batch, pages = block_table.shape
        self._tensor(block_table, (batch, pages), torch.int32, "block_table")
        self._tensor(kv_len, (batch,), torch.int32, "kv_len")
        if weights is not None:
            self._tensor(weights, (n_pages, self.n_kv_heads, self.page_size), torch.float32, "weights")
        s = k_pages.stride()
        fields = _Cache(k_pages.data_ptr(), v_pages.data_ptr(), s[0], s[1], s[2],
                        None if weights is None else weights.data_ptr(), block_table.data_ptr(), kv_len.data_ptr(),
                        n_pages, pages, batch)
        return PagedCache(fields, (k_pages, v_pages, block_table, kv_len, weights), batch, pages * self.page_size, *self._key,
                          scales, k_scales, v_scales)

    def _shapes(self, B, n):
        return (B, n, self.n_q_heads, self.head_dim), (B, n, self.n_kv_heads, self.head_dim)

    def qk_norm_rope(self, q, k, q_out, k_out, rope, pos, g_q=None, g_k=None, n_new=None, stream=None):
        """``prism_qk_norm_rope``: q, q_out [B, n, Hq, D]; k, k_out [B, n, Hkv, D]
        (strided but for D); rope fp32 [positions, 2, D / 2]; pos, n_new int32 [B]."""
        B, n = q.shape[:2]
        sq, sk = self._shapes(B, n)
        self._pack(sq, sk, q, k, None, q_out, k_out, rope, pos, g_q, g_k, n_new)
        self._check(self.lib.prism_qk_norm_rope(self.h, self._rows_at, self._stream(stream)))

    def qk_norm_rope_backward(self, dq_out, dk_out, q, k, dq, dk, rope, pos, g_q=None, g_k=None, dg_q=None, dg_k=None,
                              n_new=None, stream=None):
        """``prism_qk_norm_rope_backward``: the gradients dq, dk (zeros past
        n_new) and dg_q, dg_k (fp32 [D]) from those of the outputs and the
        forward's inputs."""
        B, n = q.shape[:2]
        sq, sk = self._shapes(B, n)
        self._pack(sq, sk, q, k, None, None, None, rope, pos, g_q, g_k, n_new)
        heads, tensor, f32 = self._heads, self._tensor, torch.float32
        _GRADS.pack_into(
            self._grads, 0, *heads(dq_out, sq, "dq_out"), *heads(dk_out, sk, "dk_out"), *heads(dq, sq, "dq"), *heads(dk, sk, "dk"),
            0 if dg_q is None else tensor(dg_q, self._dims, f32, "dg_q"), 0 if dg_k is None else tensor(dg_k, self._dims, f32, "dg_k"))
        self._check(self.lib.prism_qk_norm_rope_backward(self.h, self._rows_at, self._grads_at, self._stream(stream)))

    def append(self, cache, q, k, v, q_out, rope, g_q=None, g_k=None, pos=None, n_new=None, stream=None):
        """``prism_paged_append``: q, q_out [B, n, Hq, D]; k, v [B, n, Hkv, D].
        Rows i < n_new[b] go to slots kv_len[b] + i, at positions pos[b] + i (pos
        None: their slots).  kv_len is not advanced.  A cache held in 8 bits takes the
        keys and values quantised (``prism_paged_append_codes``)."""
        ref = self._bound(cache)
        sq, sk = self._shapes(cache.batch, q.shape[1])
        self._pack(sq, sk, q, k, v, q_out, None, rope, pos, g_q, g_k, n_new)
        if cache.scales is not None:
            self._check(self.lib.prism_paged_append_codes(self.h, ref, cache.scales_ref, self._rows_at, self._stream(stream)))
        else:
            self._check(self.lib.prism_paged_append(self.h, ref, self._rows_at, self._stream(stream)))

    def attend(self, cache, q, out, lse=None, added=1, stream=None, window=None, sinks=0):
        """``prism_paged_attend``: q, out [B, Hq, D]; lse fp32 [B, Hq] or None;
        over kv_len[b] + added rows; with ``window`` over the last ``window`` and the
        first ``sinks`` of them (``prism_paged_attend_window``).  A cache with weights
        accumulates them; one held in 8 bits is read as it is
        (``prism_paged_attend_codes``)."""
        ref = self._bound(cache)
        shape = (cache.batch, self.n_q_heads, self.head_dim)
        q, out = self._tensor(q, shape, self.tdtype, "q"), self._tensor(out, shape, self.tdtype, "out")
        lse = None if lse is None else self._tensor(lse, shape[:2], torch.float32, "lse")
        if window is None:
            if sinks:
                raise ValueError("sinks without a window")
            if cache.scales_ref is None:
                self._check(self.lib.prism_paged_attend(self.h, ref, added, q, out, lse, self._stream(stream)))
                return
            window = -1
        elif window < 0:
            raise ValueError("window is negative")
        window, sinks = min(window, 0x7FFFFFFF), min(sinks, 0x7FFFFFFF)
        if cache.scales_ref is None:
            self._check(self.lib.prism_paged_attend_window(self.h, ref, added, window, sinks, q, out, lse, self._stream(stream)))
        else:
            self._check(self.lib.prism_paged_attend_codes(self.h, ref, cache.scales_ref, added, window, sinks, q, out, lse, self._stream(stream)))

    def read(self, cache, k_out, v_out, start=None, n_rows=None, stream=None):
        """``prism_paged_read_codes``: rows start[b] + i, i < n_rows[b], of a cache held
        in 8 bits, in the handle's type; k_out, v_out [B, n, Hkv, D] (strided but for
        D); start, n_rows int32 [B] (None: 0 and n).  Rows past n_rows[b] keep what
        they hold."""
        ref = self._bound(cache)
        if cache.scales is None:
            raise ValueError("read: the cache is not held in 8 bits")
        B, n = cache.batch, k_out.shape[1]
        shape = (B, n, self.n_kv_heads, self.head_dim)
        _HEADS2.pack_into(self._kv_rows, 0, *self._heads(k_out, shape, "k_out"), *self._heads(v_out, shape, "v_out"))
        self._check(self.lib.prism_paged_read_codes(
            self.h, ref, cache.scales_ref, None if start is None else self._tensor(start, (B,), torch.int32, "start"),
            None if n_rows is None else self._tensor(n_rows, (B,), torch.int32, "n_rows"), n, self._k_rows_at, self._v_rows_at,
            self._stream(stream)))

    def evict(self, src, dst, kept, sinks=0, recent=0, stream=None):
        """``prism_paged_evict``: the rows of ``src`` to keep go, in order, to the
        pages of ``dst``; ``kept`` int32 [B, Hkv, budget] receives their slots.  Not
        for caches held in 8 bits, which have no weights."""
        rs, rd = self._bound(src), self._bound(dst)
        if src.scales is not None or dst.scales is not None:
            raise ValueError("evict: caches held in 8 bits are not evicted from")
        if kept.dim() != 3:
            raise ValueError("kept: expected three dimensions")
        budget = kept.shape[2]
        at = self._tensor(kept, (src.batch, self.n_kv_heads, budget), torch.int32, "kept")
        self._check(self.lib.prism_paged_evict(self.h, rs, rd, budget, sinks, recent, at, self._stream(stream)))

    def status(self, stream=None) -> int:
        """Synchronise; the device error word (0 when clean), cleared."""
        flags = _i32(0)
        st = self.lib.prism_paged_status(self.h, self._stream(stream), ctypes.byref(flags))
        if st not in (0, 7):
            self._check(st)
        return int(flags.value)

    def close(self):
        if getattr(self, "h", None):
            self.lib.prism_paged_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
