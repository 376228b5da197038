"""Binding of the paged-cache entry points (``ds_page_update``, ``ds_qk_norm_rope``, ``ds_attn_paged``).

Each of them exists twice: as a plan, an object made once from the tensors of a loop's call (arguments checked,
pointers and strides written down) whose ``launch`` only enqueues the kernels, and as a function that makes a plan
and launches it.  A plan keeps references to its tensors; what they contain is read at every launch.  The launch goes
to the tensors' device, on ``stream`` or that device's current stream, and may be captured into a CUDA graph; the plan
has to live as long as the graph.  Launches of one plan, and graphs that hold one, write the same results and share a
workspace: they must not overlap.  Calls that may overlap need a plan each.

Results and workspaces that are not given are allocated on the stream that is current when the plan (or function) is
called.  Their memory may have been freed there a moment ago with kernels still pending on it, so a launch on another stream
first waits for what that stream had been given by then; the caller orders the inputs, and whoever reads the results.  A graph
cannot hold that wait: one that is captured on another stream must first be replayed when that work is over (entering
``torch.cuda.graph`` waits for it; ``CUDAGraph.capture_begin`` alone does not).
"""
from __future__ import annotations

import ctypes

import torch

from . import DsError, DS_OK, _dtype_code, lib

_P, _I32, _I64, _F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class PageParams(ctypes.Structure):
    _fields_ = [("B", _I32), ("page_size", _I32), ("max_pages", _I32), ("n_pages", _I32), ("max_rows", _I32),
                ("kv_len", _P), ("n_new", _P), ("done", _P), ("block_table", _P), ("table_stride", _I64),
                ("free_list", _P), ("free_cnt", _P), ("kv_len_out", _P), ("free_cnt_out", _P), ("row_start", _P),
                ("positions", _P), ("slot_map", _P), ("status", _P)]


class RopeTableStruct(ctypes.Structure):
    _fields_ = [("rotary_dim", _I32), ("interleaved", _I32), ("mscale", _F32), ("reserved", _I32),
                ("turn", ctypes.c_uint64 * 128)]


class QkParams(ctypes.Structure):
    _fields_ = [("N", _I32), ("Hq", _I32), ("Hkv", _I32), ("D", _I32), ("dtype", _I32), ("page_size", _I32),
                ("n_pages", _I32), ("eps", _F32), ("n_rows", _P), ("q", _P), ("k", _P), ("v", _P),
                ("q_stride", _I64 * 2), ("kv_stride", _I64 * 2), ("q_weight", _P), ("k_weight", _P),
                ("positions", _P), ("rope", _P), ("q_out", _P), ("k_out", _P), ("v_out", _P),
                ("q_out_stride", _I64 * 2), ("kv_out_stride", _I64 * 2), ("k_cache", _P), ("v_cache", _P),
                ("cache_stride", _I64 * 3), ("slot_map", _P), ("status", _P)]


class PagedParams(ctypes.Structure):
    _fields_ = [("B", _I32), ("Hq", _I32), ("Hkv", _I32), ("D", _I32), ("dtype", _I32), ("N", _I32),
                ("max_q", _I32), ("max_len", _I32), ("page_size", _I32), ("max_pages", _I32), ("n_pages", _I32),
                ("causal", _I32), ("window", _I32), ("sinks", _I32), ("scale", _F32), ("row_start", _P),
                ("kv_len", _P), ("block_table", _P), ("table_stride", _I64), ("q", _P), ("q_stride", _I64 * 2),
                ("k_cache", _P), ("v_cache", _P), ("cache_stride", _I64 * 3), ("out", _P), ("out_stride", _I64 * 2),
                ("lse", _P), ("workspace", _P), ("workspace_bytes", ctypes.c_size_t), ("status", _P)]


ENTRY_POINTS = [("ds_page_update", PageParams), ("ds_qk_norm_rope", QkParams), ("ds_attn_paged", PagedParams)]


def _one_device(**tensors):
    """All tensors on one CUDA device; returns it."""
    dev = None
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("all tensors must live on a CUDA device")
        if dev is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the other tensors on {dev}")
        dev = t.device
    return dev


def _int_array(name, t, numel, dtype=torch.int32):
    if t is None:
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if not t.is_contiguous() or t.numel() < numel:
        raise ValueError(f"{name} must be contiguous with at least {numel} elements")


def _status_word(t):
    if t is not None and (t.element_size() != 4 or t.is_floating_point() or t.numel() < 1):
        raise TypeError("status must be a 32-bit integer word")


def _heads(name, t, shape, dtype):
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.stride(-1) != 1:
        raise ValueError(f"the head dimension of {name} must be contiguous")


def _cache(k_cache, v_cache, Hkv, D, dtype):
    """(pages, page size) of caches [pages, Hkv, page_size, D], in any order in memory (strides)."""
    if k_cache.dim() != 4:
        raise ValueError("the caches must be [pages, Hkv, page_size, D]")
    n_pages, _, ps, _ = k_cache.shape
    _heads("k_cache", k_cache, (n_pages, Hkv, ps, D), dtype)
    _heads("v_cache", v_cache, (n_pages, Hkv, ps, D), dtype)
    if k_cache.stride() != v_cache.stride():
        raise ValueError("k_cache and v_cache must share strides")
    return n_pages, ps


def _ptr(t):
    return None if t is None else t.data_ptr()


# The stream's handle and the device without the objects around them: a launch costs the host about as much as these.
def _raw_stream(index):
    return torch._C._cuda_getCurrentRawStream(index)


def _current_device():
    return torch._C._cuda_getDevice()


def _capturing(stream):
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _Plan:
    _name = ""

    def _ready(self, params, device, keep, own=()):
        """``own``: tensors allocated by the plan, on the stream that is current now."""
        self._params, self._keep, self.device = params, keep, device
        self._ref, self._fn = ctypes.byref(params), getattr(lib(), self._name)
        self._index = device.index
        self._own = tuple(t for t in own if t is not None)
        self._own_stream, self._own_event = torch.cuda.current_stream(device), None
        self._own_raw = self._own_stream.cuda_stream
        if self._own and not _capturing(self._own_stream):
            self._own_event = self._own_stream.record_event()

    def _wait_for_own(self, stream):
        """Orders ``stream`` behind whatever used the memory of the plan's own tensors before it had them."""
        if self._own_event is not None:
            if not _capturing(stream):
                stream.wait_event(self._own_event)
        elif _capturing(stream) and _capturing(self._own_stream):      # made within the capture, launched on a fork of it
            stream.wait_event(self._own_stream.record_event())

    def _enqueue(self, stream):
        if stream is None:
            raw = _raw_stream(self._index)
        elif stream.device != self.device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {self.device}")
        else:
            raw = stream.cuda_stream
        foreign = raw != self._own_raw and self._own
        if foreign:
            if stream is None:
                stream = torch.cuda.current_stream(self._index)
            self._wait_for_own(stream)
        if _current_device() == self._index:
            rc = self._fn(self._ref, raw)
        else:
            with torch.cuda.device(self._index):
                rc = self._fn(self._ref, raw)
        if rc != DS_OK:
            raise DsError(rc, self._name)
        if foreign:      # the allocator must not hand these out again before this stream is done
            for t in self._own:
                t.record_stream(stream)


class RopeTable:
    """Rotary frequencies (``ds_rope_table_init``), worked out once and passed with every ``ds_qk_norm_rope``.

    rotary_dim: how much of a head is rotated; interleaved: pairs (2d, 2d + 1) instead of (d, d + rotary_dim / 2);
    scaling: None, "linear", "ntk" or "yarn" (by parts; needs orig_len, the original context) with ``factor``."""

    _SCALINGS = {None: 0, "none": 0, "linear": 1, "ntk": 2, "yarn": 3}

    def __init__(self, rotary_dim: int, theta: float = 10000.0, interleaved: bool = False, scaling=None,
                 factor: float = 1.0, orig_len: float = 0, beta_fast: float = 32.0, beta_slow: float = 1.0):
        if scaling not in self._SCALINGS:
            raise ValueError(f"unknown scaling {scaling!r}")
        self.struct = RopeTableStruct()
        rc = lib().ds_rope_table_init(ctypes.byref(self.struct), int(rotary_dim), int(bool(interleaved)), float(theta),
                                      self._SCALINGS[scaling], float(factor), float(orig_len), float(beta_fast),
                                      float(beta_slow))
        if rc != DS_OK:
            raise DsError(rc, "ds_rope_table_init")


class PageUpdatePlan(_Plan):
    """``ds_page_update`` on fixed tensors.  kv_len, n_new int32 [B]; done uint8/bool [B] or None; block_table int32
    [B, max_pages] and free_list int32 [n_pages] are updated in place; free_cnt int32 [1].  The results are the
    attributes kv_len_out (kv_len itself to update in place), free_cnt_out, row_start [B + 1], positions int32 and
    slot_map int64 [max_rows]; those not given are allocated."""

    _name = "ds_page_update"

    def __init__(self, kv_len, n_new, block_table, free_list, free_cnt, page_size, max_rows=None, done=None,
                 kv_len_out=None, free_cnt_out=None, row_start=None, positions=None, slot_map=None, status=None):
        dev = _one_device(kv_len=kv_len, n_new=n_new, block_table=block_table, free_list=free_list, free_cnt=free_cnt,
                          done=done, kv_len_out=kv_len_out, free_cnt_out=free_cnt_out, row_start=row_start,
                          positions=positions, slot_map=slot_map, status=status)
        B = kv_len.numel()
        if max_rows is None:
            sizes = [t.numel() for t in (positions, slot_map) if t is not None]
            if not sizes:
                raise ValueError("max_rows is needed when neither positions nor slot_map is given")
            max_rows = min(sizes)
        given = (kv_len_out, free_cnt_out, row_start, positions, slot_map)
        i32 = dict(dtype=torch.int32, device=dev)
        self.kv_len_out = torch.empty(B, **i32) if kv_len_out is None else kv_len_out
        self.free_cnt_out = torch.empty(1, **i32) if free_cnt_out is None else free_cnt_out
        self.row_start = torch.empty(B + 1, **i32) if row_start is None else row_start
        self.positions = torch.empty(max_rows, **i32) if positions is None else positions
        self.slot_map = torch.empty(max_rows, dtype=torch.int64, device=dev) if slot_map is None else slot_map
        self.block_table, self.free_list = block_table, free_list
        for name, t, n in (("kv_len", kv_len, B), ("n_new", n_new, B), ("free_cnt", free_cnt, 1),
                           ("kv_len_out", self.kv_len_out, B), ("free_cnt_out", self.free_cnt_out, 1),
                           ("row_start", self.row_start, B + 1), ("positions", self.positions, max_rows),
                           ("free_list", free_list, 1)):
            _int_array(name, t, n)
        _int_array("slot_map", self.slot_map, max_rows, torch.int64)
        _status_word(status)
        if done is not None and (done.dtype not in (torch.uint8, torch.bool) or not done.is_contiguous() or done.numel() < B):
            raise ValueError("done must be uint8 or bool [B]")
        if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != B or (
                block_table.shape[1] > 1 and block_table.stride(1) != 1):
            raise ValueError("block_table must be int32 [B, max_pages] with contiguous rows")
        p = PageParams()
        p.B, p.page_size, p.max_pages, p.n_pages = B, int(page_size), block_table.shape[1], free_list.numel()
        p.max_rows, p.table_stride = int(max_rows), max(block_table.stride(0), block_table.shape[1]) if B < 2 else block_table.stride(0)
        p.kv_len, p.n_new, p.done, p.block_table = _ptr(kv_len), _ptr(n_new), _ptr(done), _ptr(block_table)
        p.free_list, p.free_cnt = _ptr(free_list), _ptr(free_cnt)
        p.kv_len_out, p.free_cnt_out = _ptr(self.kv_len_out), _ptr(self.free_cnt_out)
        p.row_start, p.positions, p.slot_map = _ptr(self.row_start), _ptr(self.positions), _ptr(self.slot_map)
        p.status = _ptr(status)
        results = (self.kv_len_out, self.free_cnt_out, self.row_start, self.positions, self.slot_map)
        self._ready(p, dev, (kv_len, n_new, done, free_cnt, status),
                    [r for r, g in zip(results, given) if g is None])

    def launch(self, stream=None):
        self._enqueue(stream)
        return self


def ds_page_update(kv_len, n_new, block_table, free_list, free_cnt, page_size, max_rows=None, done=None,
                   kv_len_out=None, free_cnt_out=None, row_start=None, positions=None, slot_map=None, status=None,
                   stream=None):
    """One step's bookkeeping of the paged cache; see ``PageUpdatePlan`` for the arguments.  Returns a dict with
    kv_len_out, free_cnt_out, row_start, positions, slot_map."""
    plan = PageUpdatePlan(kv_len, n_new, block_table, free_list, free_cnt, page_size, max_rows, done, kv_len_out,
                          free_cnt_out, row_start, positions, slot_map, status)
    plan.launch(stream)
    return {n: getattr(plan, n) for n in ("kv_len_out", "free_cnt_out", "row_start", "positions", "slot_map")}


class QkNormRopePlan(_Plan):
    """``ds_qk_norm_rope`` on fixed tensors.  q [N, Hq, D], k and v [N, Hkv, D] (e.g. slices of a fused projection's
    output); positions int32 [N]; rope a RopeTable; q_weight, k_weight [D] or None (no norm); caches
    [pages, Hkv, page_size, D] of any strides with slot_map int64 [N]; k_out, v_out [N, Hkv, D]; n_rows an int32
    device word.  q_out is allocated when not given; it may be q itself, as k_out and v_out may be k and v."""

    _name = "ds_qk_norm_rope"

    def __init__(self, q, k, v, positions, rope, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None,
                 v_out=None, k_cache=None, v_cache=None, slot_map=None, n_rows=None, status=None):
        dev = _one_device(q=q, k=k, v=v, positions=positions, q_weight=q_weight, k_weight=k_weight, q_out=q_out,
                          k_out=k_out, v_out=v_out, k_cache=k_cache, v_cache=v_cache, slot_map=slot_map, n_rows=n_rows,
                          status=status)
        if q.dim() != 3 or k.dim() != 3:
            raise ValueError("q must be [N, Hq, D] and k, v [N, Hkv, D]")
        N, Hq, D = q.shape
        Hkv, dt = k.shape[1], q.dtype
        self.q_out = torch.empty((N, Hq, D), dtype=dt, device=dev) if q_out is None else q_out
        self.k_out, self.v_out = k_out, v_out
        _heads("q", q, (N, Hq, D), dt)
        _heads("q_out", self.q_out, (N, Hq, D), dt)
        for name, t in (("k", k), ("v", v), ("k_out", k_out), ("v_out", v_out)):
            if t is not None:
                _heads(name, t, (N, Hkv, D), dt)
        if k.stride() != v.stride():
            raise ValueError("k and v must share strides")
        if (k_out is None) != (v_out is None) or (k_cache is None) != (v_cache is None):
            raise ValueError("k_out and v_out, k_cache and v_cache come in pairs")
        if k_out is not None and k_out.stride() != v_out.stride():
            raise ValueError("k_out and v_out must share strides")
        for name, t in (("q_weight", q_weight), ("k_weight", k_weight)):
            if t is not None and (t.dtype != dt or not t.is_contiguous() or t.numel() != D):
                raise ValueError(f"{name} must be {dt} [D]")
        if not isinstance(rope, RopeTable):
            raise TypeError("rope must be a RopeTable")
        _int_array("positions", positions, N)
        _int_array("n_rows", n_rows, 1)
        _status_word(status)
        p = QkParams()
        p.N, p.Hq, p.Hkv, p.D, p.dtype, p.eps = N, Hq, Hkv, D, _dtype_code(q), float(eps)
        if k_cache is not None:
            if slot_map is None:
                raise ValueError("a cache needs a slot_map")
            _int_array("slot_map", slot_map, N, torch.int64)
            p.n_pages, p.page_size = _cache(k_cache, v_cache, Hkv, D, dt)
            p.k_cache, p.v_cache, p.slot_map = _ptr(k_cache), _ptr(v_cache), _ptr(slot_map)
            p.cache_stride[:] = k_cache.stride()[:3]
        p.n_rows, p.q, p.k, p.v = _ptr(n_rows), _ptr(q), _ptr(k), _ptr(v)
        p.q_stride[:], p.kv_stride[:], p.q_out_stride[:] = q.stride()[:2], k.stride()[:2], self.q_out.stride()[:2]
        p.q_weight, p.k_weight, p.positions = _ptr(q_weight), _ptr(k_weight), _ptr(positions)
        p.rope, p.q_out, p.k_out, p.v_out = ctypes.addressof(rope.struct), _ptr(self.q_out), _ptr(k_out), _ptr(v_out)
        if k_out is not None:
            p.kv_out_stride[:] = k_out.stride()[:2]
        p.status = _ptr(status)
        self._ready(p, dev, (q, k, v, positions, rope, q_weight, k_weight, k_cache, v_cache, slot_map, n_rows, status),
                    [self.q_out if q_out is None else None])

    def launch(self, stream=None):
        self._enqueue(stream)
        return self.q_out


def ds_qk_norm_rope(q, k, v, positions, rope, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None,
                    v_out=None, k_cache=None, v_cache=None, slot_map=None, n_rows=None, status=None, stream=None):
    """Norm of every query and key head, rotary position, and K and V written to k_out/v_out and the paged cache; see
    ``QkNormRopePlan`` for the arguments.  Returns q_out."""
    return QkNormRopePlan(q, k, v, positions, rope, q_weight, k_weight, eps, q_out, k_out, v_out, k_cache, v_cache,
                          slot_map, n_rows, status).launch(stream)


def _paged_params(q, k_cache, v_cache, block_table, kv_len, scale, row_start, max_q, max_len, causal, window, sinks,
                  out, lse, status):
    if q.dim() != 3:
        raise ValueError("q must be [N, Hq, D]")
    N, Hq, D = q.shape
    B, Hkv = kv_len.numel(), k_cache.shape[1]
    _heads("q", q, (N, Hq, D), q.dtype)
    if out is not None:
        _heads("out", out, (N, Hq, D), q.dtype)
    _int_array("kv_len", kv_len, B)
    _int_array("row_start", row_start, B + 1)
    _status_word(status)
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != B or (
            block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table must be int32 [B, max_pages] with contiguous rows")
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (N, Hq)):
        raise ValueError("lse must be contiguous f32 [N, Hq]")
    p = PagedParams()
    p.n_pages, p.page_size = _cache(k_cache, v_cache, Hkv, D, q.dtype)
    p.B, p.Hq, p.Hkv, p.D, p.dtype, p.N = B, Hq, Hkv, D, _dtype_code(q), N
    p.max_q, p.max_len, p.max_pages = int(max_q), int(max_len), block_table.shape[1]
    p.causal, p.window, p.sinks, p.scale = int(bool(causal)), int(window), int(sinks), float(scale)
    p.row_start, p.kv_len, p.block_table = _ptr(row_start), _ptr(kv_len), _ptr(block_table)
    p.table_stride = block_table.stride(0) if B > 1 else max(block_table.stride(0), block_table.shape[1])
    p.q, p.k_cache, p.v_cache = _ptr(q), _ptr(k_cache), _ptr(v_cache)
    p.q_stride[:], p.cache_stride[:] = q.stride()[:2], k_cache.stride()[:3]
    if out is not None:
        p.out = _ptr(out)
        p.out_stride[:] = out.stride()[:2]
    p.lse, p.status = _ptr(lse), _ptr(status)
    return p


def ds_attn_paged_workspace(q, k_cache, v_cache, block_table, kv_len, scale, row_start=None, max_q=1, max_len=0,
                            causal=True, window=0, sinks=0) -> int:
    """Bytes of workspace the call wants (0: none)."""
    _one_device(q=q, k_cache=k_cache, v_cache=v_cache, block_table=block_table, kv_len=kv_len, row_start=row_start)
    p = _paged_params(q, k_cache, v_cache, block_table, kv_len, scale, row_start, max_q, max_len, causal, window, sinks,
                      None, None, None)
    p.out = p.q     # the size does not depend on it
    p.out_stride[:] = p.q_stride[:]
    return int(lib().ds_attn_paged_workspace(ctypes.byref(p)))


class PagedAttnPlan(_Plan):
    """``ds_attn_paged`` on fixed tensors.  q [N, Hq, D]: the new rows of all sequences, packed; row_start int32
    [B + 1] (None: max_q rows each); caches [pages, Hkv, page_size, D] of any strides; block_table int32
    [B, max_pages]; kv_len int32 [B], the new rows included.  max_q and max_len (0: the table's capacity) bound what
    row_start and kv_len will hold.  causal, or bidirectional within kv_len; window > 0 hides all but the last
    ``window`` rows and the first ``sinks``.  out (like q), lse (f32 [N, Hq], optional) and workspace (uint8) are the
    caller's or allocated here: the result is the attribute ``out``."""

    _name = "ds_attn_paged"

    def __init__(self, q, k_cache, v_cache, block_table, kv_len, scale, row_start=None, max_q=1, max_len=0, causal=True,
                 window=0, sinks=0, out=None, lse=None, workspace=None, status=None):
        dev = _one_device(q=q, k_cache=k_cache, v_cache=v_cache, block_table=block_table, kv_len=kv_len,
                          row_start=row_start, out=out, lse=lse, workspace=workspace, status=status)
        self.out = torch.empty(q.shape, dtype=q.dtype, device=dev) if out is None else out
        self.lse = lse
        p = _paged_params(q, k_cache, v_cache, block_table, kv_len, scale, row_start, max_q, max_len, causal, window,
                          sinks, self.out, lse, status)
        own = [self.out if out is None else None]
        if workspace is None:
            need = int(lib().ds_attn_paged_workspace(ctypes.byref(p)))
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
                own.append(workspace)
        elif not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        if workspace is not None:
            p.workspace, p.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self._ready(p, dev, (q, k_cache, v_cache, block_table, kv_len, row_start, workspace, status), own)

    def launch(self, stream=None):
        self._enqueue(stream)
        return self.out


def ds_attn_paged(q, k_cache, v_cache, block_table, kv_len, scale, row_start=None, max_q=1, max_len=0, causal=True,
                  window=0, sinks=0, out=None, lse=None, workspace=None, status=None, stream=None):
    """Attention of the new rows of every sequence over its pages; see ``PagedAttnPlan`` for the arguments.
    Returns out [N, Hq, D]."""
    return PagedAttnPlan(q, k_cache, v_cache, block_table, kv_len, scale, row_start, max_q, max_len, causal, window,
                         sinks, out, lse, workspace, status).launch(stream)
