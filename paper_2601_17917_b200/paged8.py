"""Binding of the 8-bit paged cache (``ds_kv8_write``, ``ds_kv8_read``, ``ds_attn_paged8``): plans and functions as in ``paged.py``.

The caches are e4m3 [pages, Hkv, page_size, D] (``torch.float8_e4m3fn``, or ``torch.uint8`` holding the same bytes) of any strides, the
scales fp32 [pages, Hkv, page_size / T] of any strides: one for every T rows of a page and KV head.  T is taken from their shape."""
from __future__ import annotations

import ctypes

import torch

from . import _dtype_code, lib
from .paged import (_I32, _I64, _P, PagedParams, _cache, _heads, _int_array, _one_device, _paged_params, _Plan, _ptr,
                    _status_word)


class Kv8WriteParams(ctypes.Structure):
    _fields_ = [("B", _I32), ("Hkv", _I32), ("D", _I32), ("dtype", _I32), ("N", _I32), ("max_q", _I32), ("max_len", _I32),
                ("page_size", _I32), ("max_pages", _I32), ("n_pages", _I32), ("scale_block", _I32), ("row_start", _P),
                ("kv_len", _P), ("block_table", _P), ("table_stride", _I64), ("k", _P), ("v", _P), ("kv_stride", _I64 * 2),
                ("k_cache", _P), ("v_cache", _P), ("cache_stride", _I64 * 3), ("k_scale", _P), ("v_scale", _P),
                ("scale_stride", _I64 * 3), ("status", _P)]


class Kv8ReadParams(ctypes.Structure):
    _fields_ = [("B", _I32), ("Hkv", _I32), ("D", _I32), ("dtype", _I32), ("N", _I32), ("page_size", _I32), ("max_pages", _I32),
                ("n_pages", _I32), ("scale_block", _I32), ("out_start", _P), ("first", _P), ("kv_len", _P), ("block_table", _P),
                ("table_stride", _I64), ("k_cache", _P), ("v_cache", _P), ("cache_stride", _I64 * 3), ("k_scale", _P),
                ("v_scale", _P), ("scale_stride", _I64 * 3), ("k_out", _P), ("v_out", _P), ("out_stride", _I64 * 3),
                ("status", _P)]


class Paged8Params(ctypes.Structure):
    _fields_ = [("a", PagedParams), ("scale_block", _I32), ("k_scale", _P), ("v_scale", _P), ("scale_stride", _I64 * 3)]


ENTRY_POINTS = [("ds_kv8_write", Kv8WriteParams), ("ds_kv8_read", Kv8ReadParams), ("ds_attn_paged8", Paged8Params)]


def _codes(name, t):
    if t.dtype == torch.uint8:
        return t.view(torch.float8_e4m3fn)
    if t.dtype != torch.float8_e4m3fn:
        raise TypeError(f"{name} must be torch.float8_e4m3fn or torch.uint8")
    return t


def _scales(p, k_scale, v_scale, n_pages, Hkv, page_size):
    for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        if t.dtype != torch.float32:
            raise TypeError(f"{name} must be torch.float32")
        if t.dim() != 3 or tuple(t.shape[:2]) != (n_pages, Hkv) or t.shape[2] < 1 or page_size % t.shape[2]:
            raise ValueError(f"{name} must be [{n_pages}, {Hkv}, page_size / T], not {tuple(t.shape)}")
    if k_scale.shape != v_scale.shape or k_scale.stride() != v_scale.stride():
        raise ValueError("k_scale and v_scale must share shape and strides")
    p.scale_block = page_size // k_scale.shape[2]
    p.k_scale, p.v_scale = _ptr(k_scale), _ptr(v_scale)
    p.scale_stride[:] = k_scale.stride()


def _table(p, block_table, B):
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != B or (
            block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table must be int32 [B, max_pages] with contiguous rows")
    p.block_table, p.max_pages = _ptr(block_table), block_table.shape[1]
    p.table_stride = block_table.stride(0) if B > 1 else max(block_table.stride(0), block_table.shape[1])


def _pool(p, k_cache, v_cache, k_scale, v_scale, Hkv, D):
    k_cache, v_cache = _codes("k_cache", k_cache), _codes("v_cache", v_cache)
    p.n_pages, p.page_size = _cache(k_cache, v_cache, Hkv, D, torch.float8_e4m3fn)
    _scales(p, k_scale, v_scale, p.n_pages, Hkv, p.page_size)
    p.k_cache, p.v_cache = _ptr(k_cache), _ptr(v_cache)
    p.cache_stride[:] = k_cache.stride()[:3]


class Kv8WritePlan(_Plan):
    """``ds_kv8_write`` on fixed tensors.  k and v [N, Hkv, D]: the packed new rows of all sequences (e.g. ``k_out`` and ``v_out``
    of ``ds_qk_norm_rope``), which are the last rows of each; row_start int32 [B + 1] (None: max_q rows each); block_table int32
    [B, max_pages]; kv_len int32 [B], the new rows included.  max_q and max_len (0: the table's capacity) bound what row_start and
    kv_len will hold.  Caches and scales are updated in place."""

    _name = "ds_kv8_write"

    def __init__(self, k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, row_start=None, max_q=1, max_len=0,
                 status=None):
        dev = _one_device(k=k, v=v, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, block_table=block_table,
                          kv_len=kv_len, row_start=row_start, status=status)
        if k.dim() != 3:
            raise ValueError("k and v must be [N, Hkv, D]")
        N, Hkv, D = k.shape
        _heads("k", k, (N, Hkv, D), k.dtype)
        _heads("v", v, (N, Hkv, D), k.dtype)
        if k.stride() != v.stride():
            raise ValueError("k and v must share strides")
        B = kv_len.numel()
        _int_array("kv_len", kv_len, B)
        _int_array("row_start", row_start, B + 1)
        _status_word(status)
        p = Kv8WriteParams()
        p.B, p.Hkv, p.D, p.dtype, p.N = B, Hkv, D, _dtype_code(k), N
        p.max_q, p.max_len = int(max_q), int(max_len)
        _pool(p, k_cache, v_cache, k_scale, v_scale, Hkv, D)
        _table(p, block_table, B)
        p.row_start, p.kv_len, p.k, p.v = _ptr(row_start), _ptr(kv_len), _ptr(k), _ptr(v)
        p.kv_stride[:] = k.stride()[:2]
        p.status = _ptr(status)
        self._ready(p, dev, (k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, row_start, status))

    def launch(self, stream=None):
        self._enqueue(stream)
        return self


def ds_kv8_write(k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, row_start=None, max_q=1, max_len=0, status=None,
                 stream=None):
    """Quantises the new rows of every sequence into its pages; see ``Kv8WritePlan`` for the arguments."""
    Kv8WritePlan(k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, row_start, max_q, max_len, status).launch(stream)


class Kv8ReadPlan(_Plan):
    """``ds_kv8_read`` on fixed tensors: rows first[b] .. (int32 [B]; None: from row 0) of every sequence in bf16 or fp32.

    k_out and v_out [N, Hkv, D] with out_start int32 [B + 1]: rows out_start[b] .. out_start[b + 1] - 1 are sequence b's; or
    [B, L, Hkv, D] without: up to L rows of each, what lies behind a sequence's last row is left as it is."""

    _name = "ds_kv8_read"

    def __init__(self, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, k_out, v_out, out_start=None, first=None,
                 status=None):
        dev = _one_device(k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, block_table=block_table, kv_len=kv_len,
                          k_out=k_out, v_out=v_out, out_start=out_start, first=first, status=status)
        B, dense = kv_len.numel(), out_start is None
        if k_out.dim() != (4 if dense else 3) or (dense and k_out.shape[0] != B):
            raise ValueError("k_out and v_out must be [N, Hkv, D] with out_start, [B, L, Hkv, D] without")
        N, Hkv, D = k_out.shape[-3:]
        for name, t in (("k_out", k_out), ("v_out", v_out)):
            _heads(name, t, k_out.shape, k_out.dtype)
        if k_out.stride() != v_out.stride():
            raise ValueError("k_out and v_out must share strides")
        _int_array("kv_len", kv_len, B)
        _int_array("out_start", out_start, B + 1)
        _int_array("first", first, B)
        _status_word(status)
        p = Kv8ReadParams()
        p.B, p.Hkv, p.D, p.dtype, p.N = B, Hkv, D, _dtype_code(k_out), N
        _pool(p, k_cache, v_cache, k_scale, v_scale, Hkv, D)
        _table(p, block_table, B)
        p.out_start, p.first, p.kv_len = _ptr(out_start), _ptr(first), _ptr(kv_len)
        p.k_out, p.v_out = _ptr(k_out), _ptr(v_out)
        p.out_stride[:] = k_out.stride()[:3] if dense else (0, *k_out.stride()[:2])
        p.status = _ptr(status)
        self.k_out, self.v_out = k_out, v_out
        self._ready(p, dev, (k_cache, v_cache, k_scale, v_scale, block_table, kv_len, out_start, first, status))

    def launch(self, stream=None):
        self._enqueue(stream)
        return self.k_out, self.v_out


def ds_kv8_read(k_cache, v_cache, k_scale, v_scale, block_table, kv_len, k_out, v_out, out_start=None, first=None, status=None,
                stream=None):
    """Rows of the 8-bit cache in bf16 or fp32; see ``Kv8ReadPlan`` for the arguments.  Returns k_out, v_out."""
    return Kv8ReadPlan(k_cache, v_cache, k_scale, v_scale, block_table, kv_len, k_out, v_out, out_start, first, status).launch(stream)


def _paged8_params(q, k_cache, v_cache, k_scale, v_scale, *args):
    k_cache, v_cache = _codes("k_cache", k_cache), _codes("v_cache", v_cache)
    p = Paged8Params()
    p.a = _paged_params(q, k_cache, v_cache, *args, cache_dtype=torch.float8_e4m3fn)
    _scales(p, k_scale, v_scale, p.a.n_pages, p.a.Hkv, p.a.page_size)
    return p


def ds_attn_paged8_workspace(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, scale, row_start=None, max_q=1, max_len=0,
                             causal=True, window=0, sinks=0) -> int:
    """Bytes of workspace the call wants (0: none)."""
    _one_device(q=q, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, block_table=block_table, kv_len=kv_len,
                row_start=row_start)
    p = _paged8_params(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, scale, row_start, max_q, max_len, causal, window,
                       sinks, None, None, None)
    p.a.out = p.a.q     # the size does not depend on it
    p.a.out_stride[:] = p.a.q_stride[:]
    return int(lib().ds_attn_paged8_workspace(ctypes.byref(p)))


class PagedAttn8Plan(_Plan):
    """``ds_attn_paged8`` on fixed tensors: ``PagedAttnPlan`` with an 8-bit cache and its scales.  q [N, Hq, D] and out are bf16
    or fp32; the other arguments are those of ``PagedAttnPlan``."""

    _name = "ds_attn_paged8"

    def __init__(self, q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, scale, row_start=None, max_q=1, max_len=0,
                 causal=True, window=0, sinks=0, out=None, lse=None, workspace=None, status=None):
        dev = _one_device(q=q, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, block_table=block_table,
                          kv_len=kv_len, row_start=row_start, out=out, lse=lse, workspace=workspace, status=status)
        self.out = torch.empty(q.shape, dtype=q.dtype, device=dev) if out is None else out
        self.lse = lse
        p = _paged8_params(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, scale, row_start, max_q, max_len, causal,
                           window, sinks, self.out, lse, status)
        own = [self.out if out is None else None]
        if workspace is None:
            need = int(lib().ds_attn_paged8_workspace(ctypes.byref(p)))
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
                own.append(workspace)
        elif not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        if workspace is not None:
            p.a.workspace, p.a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self._ready(p, dev, (q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, row_start, workspace, status), own)

    def launch(self, stream=None):
        self._enqueue(stream)
        return self.out


def ds_attn_paged8(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, scale, row_start=None, max_q=1, max_len=0,
                   causal=True, window=0, sinks=0, out=None, lse=None, workspace=None, status=None, stream=None):
    """Attention of the new rows of every sequence over its pages of an 8-bit cache; see ``PagedAttn8Plan`` for the arguments.
    Returns out [N, Hq, D]."""
    return PagedAttn8Plan(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, scale, row_start, max_q, max_len, causal,
                          window, sinks, out, lse, workspace, status).launch(stream)
