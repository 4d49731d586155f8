"""ctypes binding of the attention entry points of include/bsm.h: ragged sequences with their
gradient, and the paged key/value cache.

Operands are bfloat16 GPU tensors of any strides whose last dimension is contiguous:
(tokens, heads, dim), or (batch, rows, heads, dim) for padded batches (a heads-first tensor is
passed transposed). Nothing is copied or computed here.
"""

from __future__ import annotations

import ctypes
import itertools
import math
import struct
import threading

import numpy as np
import torch

from . import bsm as _b
from .bsm import _arr, _check, _schedule_code, _stream_of, bsm_topology

_vp, _i64, _i32, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float

# bits of a plan's "forms": which kernels its calls run
BSM_ATTENTION_HALF_FORWARD, BSM_ATTENTION_HALF_DQ, BSM_ATTENTION_HALF_KEYS = 1, 2, 4
BSM_ATTENTION_LONG_STEPS, BSM_ATTENTION_DQ_PARTS, BSM_ATTENTION_KEY_PARTS = 8, 16, 32


class bsm_heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("seq", _i64), ("row", _i64), ("head", _i64)]


class bsm_cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("n_pages", _i64), ("page_stride", _i64),
                ("row_stride", _i64), ("head_stride", _i64), ("page_size", _i32),
                ("heads", _i32), ("head_dim", _i32), ("reserved", _i32)]


class bsm_attention_stats(ctypes.Structure):
    _fields_ = [("batch", _i64), ("total_q", _i64), ("total_kv", _i64), ("q_units", _i64),
                ("kv_units", _i64), ("lse_elems", _i64), ("workspace_bytes", _i64),
                ("pairs", _i64), ("heads_q", _i32), ("heads_kv", _i32), ("head_dim", _i32),
                ("causal", _i32), ("window", _i32), ("schedule", _i32), ("n_xcd", _i32),
                ("forms", _i32)]


_lib = None


def _load() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    lib = _b.load()
    P = ctypes.POINTER
    H = _vp  # bsm_heads, as _refs makes them
    c_int = ctypes.c_int
    sig = {
        "bsm_attention_plan_create": [P(_vp), P(_i32), P(_i32), P(_i64), P(_i64), _i64, _i32, _i32,
                                      _i32, _i32, _i32, c_int, P(bsm_topology), c_int],
        "bsm_attention_plan_describe": [_vp, P(bsm_attention_stats)],
        "bsm_attention_plan_destroy": [_vp],
        "bsm_attention_execute": [_vp, H, H, H, H, _vp, _f32, _vp],
        "bsm_attention_backward": [_vp, H, H, H, H, _vp, H, H, H, H, _f32, _vp, _i64, _vp],
        "bsm_cache_slots": [_vp, _vp, _i64, _i32, _i64, _vp, _i32, _vp, _i64, _vp, _vp, _vp, _vp,
                            _i64, _vp, _vp],
        "bsm_cache_append": [P(bsm_cache), H, H, _vp, _i64, _vp],
        "bsm_attention_paged": [P(bsm_cache), H, H, _vp, _i32, _vp, _vp, _i64, _i64, _i32, _i32,
                                _i32, _i32, _f32, _vp, _i64, _vp],
        "bsm_attention_paged_workspace": [_i64, _i64, _i32, _i32, _i32, _i32, _i32, c_int,
                                          P(_i64)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = c_int
    _lib = lib
    return lib


# The stream's handle without a Stream object around it (a call of these is mostly launch time).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(index, stream):
    """The handle of `stream` (None: the current one) for a call on GPU `index`."""
    if stream is not None:
        if getattr(stream, "device_index", index) != index:
            raise ValueError(f"the stream is on cuda:{stream.device_index}, the tensors are on cuda:{index}")
        return _stream_of(None, stream)
    if _raw_stream is not None:
        return _raw_stream(index)
    return torch.cuda.current_stream(index).cuda_stream


def _call(index, fn, *args) -> None:
    """Calls a C entry point with GPU `index` as the current device."""
    if torch.cuda.current_device() == index:
        status = fn(*args)
    else:
        with torch.cuda.device(index):
            status = fn(*args)
    if status:
        _check(status)


def _contiguous(t, dtype, n, name, index) -> int:
    """Pointer of a contiguous tensor of `dtype` on GPU `index` with at least n elements."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on cuda:{index}")
    if t.numel() < n:
        raise ValueError(f"{name} has {t.numel()} elements, needs {n}")
    return t.data_ptr()


def _operand(t, rows, batch, heads, dim, name, index):
    """The fields of a bsm_heads for `t`: (tokens, heads, dim) with at least `rows` tokens, or
    (batch, rows, heads, dim), on GPU `index`."""
    shape = t.shape
    n = len(shape)
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} must be bfloat16, got {t.dtype}")
    if t.get_device() != index or index < 0:
        raise ValueError(f"{name} must be a tensor on cuda:{index}, got one on {t.device}")
    if n not in (3, 4) or shape[-2] != heads or shape[-1] != dim:
        raise ValueError(f"{name} of shape {tuple(shape)} is no (tokens, {heads}, {dim}) or "
                         f"(batch, rows, {heads}, {dim})")
    stride = t.stride()
    if stride[-1] != 1 and dim > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if shape[-3] < rows or (n == 4 and shape[0] < batch):
        raise ValueError(f"{name} of shape {tuple(shape)} is shorter than the sequences "
                         f"({batch} sequences, rows up to {rows})")
    if n == 3:
        return t.data_ptr(), 0, stride[0], stride[1]
    return t.data_ptr(), *stride[:3]


class _Scratch(threading.local):
    """A thread's memory for the bsm_heads of a call, which the library reads before it returns."""

    def __init__(self):
        self.memory = (_i64 * 32)()
        self.at = ctypes.addressof(self.memory)


_scratch = _Scratch()
_FIELDS = {n: struct.Struct(f"{4 * n}q") for n in (2, 4, 8)}


def _refs(*operands):
    """Addresses of a bsm_heads for each operand's fields, good until the thread's next call."""
    n, at = len(operands), _scratch.at
    _FIELDS[n].pack_into(_scratch.memory, 0, *itertools.chain.from_iterable(operands))
    return range(at, at + 32 * n, 32)


def _ref(x):
    return ctypes.byref(x)


def _int32(**values):
    """The values as ints that the library's 32-bit arguments hold (ctypes would cut them off)."""
    for name, x in values.items():
        x = int(x)
        if not -2**31 <= x < 2**31:
            raise ValueError(f"{name} {x} must fit in 32 bits")
        yield x


# ------------------------------------------------------------------------- ragged sequences
class AttentionPlan:
    """A plan of one batch's geometry (bsm_attention_plan). Use bsm_attention_plan_create."""

    def __init__(self, handle: int, device: int, stats: bsm_attention_stats, q_end: int,
                 kv_end: int):
        self.handle = handle
        self.device = device
        self.batch = int(stats.batch)
        self.heads_q, self.heads_kv, self.head_dim = stats.heads_q, stats.heads_kv, stats.head_dim
        self.total_q, self.total_kv = int(stats.total_q), int(stats.total_kv)
        self.lse_elems, self.workspace_bytes = int(stats.lse_elems), int(stats.workspace_bytes)
        self.q_end, self.kv_end = q_end, kv_end

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.destroy()

    def destroy(self):
        if self.handle:
            h, self.handle = self.handle, None
            _check(_load().bsm_attention_plan_destroy(h))

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _q(self, t, name):
        return _operand(t, self.q_end, self.batch, self.heads_q, self.head_dim, name, self.device)

    def _kv(self, t, name):
        return _operand(t, self.kv_end, self.batch, self.heads_kv, self.head_dim, name, self.device)


def _lengths(a, n=None):
    a = np.asarray(a.cpu() if isinstance(a, torch.Tensor) else a).reshape(-1)
    if a.size and (a.max() > 2**31 - 1 or a.min() < -2**31):
        raise ValueError("sequence lengths must fit in 32 bits")
    return np.ascontiguousarray(a, dtype=np.int32)


def _first_rows(start, lengths):
    if start is None:
        return None, int(lengths.astype(np.int64).sum())
    s = np.asarray(start.cpu() if isinstance(start, torch.Tensor) else start, dtype=np.int64)
    s = np.ascontiguousarray(np.broadcast_to(s.reshape(-1), lengths.shape))
    live = lengths > 0
    return s, int((s[live] + lengths[live]).max()) if live.any() else 0


def bsm_attention_plan_create(q_len, kv_len=None, *, heads_q, heads_kv=None, head_dim,
                              causal=False, window=0, q_start=None, kv_start=None,
                              schedule="balanced", topology=None, device=0) -> AttentionPlan:
    """Plan of attention over sequences of q_len query rows and kv_len keys (default: as many).
    q_start / kv_start: first row of each sequence in the operands; None for sequences packed one
    after the other, 0 for (batch, rows, heads, dim) operands. device=-1 makes a host-only plan
    (needs a topology)."""
    lib = _load()
    q_len = _lengths(q_len)
    kv_len = q_len if kv_len is None else _lengths(kv_len)
    if q_len.shape != kv_len.shape:
        raise ValueError(f"{q_len.size} query lengths, {kv_len.size} key lengths")
    q_start, q_end = _first_rows(q_start, q_len)
    kv_start, kv_end = _first_rows(kv_start, kv_len)
    topo = None
    if topology is not None:
        topo = topology if isinstance(topology, bsm_topology) else bsm_topology(**topology)
    keep = [_arr(q_len, np.int32), _arr(kv_len, np.int32), _arr(q_start, np.int64),
            _arr(kv_start, np.int64)]
    hq, hk, dim, window, device = _int32(
        heads_q=heads_q, heads_kv=heads_q if heads_kv is None else heads_kv, head_dim=head_dim,
        window=window, device=device)
    handle = _vp()
    _check(lib.bsm_attention_plan_create(
        _ref(handle), keep[0][1], keep[1][1], keep[2][1], keep[3][1], q_len.size, hq, hk, dim,
        int(bool(causal)), window, _schedule_code(schedule),
        _ref(topo) if topo is not None else None, device))
    st = bsm_attention_stats()
    _check(lib.bsm_attention_plan_describe(handle.value, _ref(st)))
    return AttentionPlan(handle.value, device, st, q_end, kv_end)


def bsm_attention_plan_describe(plan: AttentionPlan) -> dict:
    st = bsm_attention_stats()
    _check(_load().bsm_attention_plan_describe(plan.handle, _ref(st)))
    return {name: getattr(st, name) for name, _ in st._fields_}


def bsm_attention_plan_destroy(plan: AttentionPlan) -> None:
    plan.destroy()


def _scale_of(scale, dim) -> float:
    return 1.0 / math.sqrt(dim) if scale is None else float(scale)


def bsm_attention_execute(plan: AttentionPlan, q, k, v, o, lse=None, scale=None, stream=None):
    """o = attention of q over k and v under the plan (see bsm.h); lse: None or a float32 tensor
    of heads_q * total_q elements for the rows' log-sum-exp, which the backward pass needs.
    scale: default 1 / sqrt(head_dim). Returns o."""
    fn = _load().bsm_attention_execute
    refs = _refs(plan._q(q, "q"), plan._kv(k, "k"), plan._kv(v, "v"), plan._q(o, "o"))
    dev = plan.device
    lp = None if lse is None else _contiguous(lse, torch.float32, plan.lse_elems, "lse", dev)
    _call(dev, fn, plan.handle, *refs, lp, _scale_of(scale, plan.head_dim), _stream(dev, stream))
    return o


def bsm_attention_backward(plan: AttentionPlan, q, k, v, o, lse, dout, dq, dk, dv, scale=None,
                           workspace=None, stream=None):
    """Gradients of bsm_attention_execute: dq, dk and dv from q, k, v, its o and lse, and dout
    (see bsm.h). workspace: None (allocated for the call on the current stream; a call with a stream
    of its own brings its own) or a tensor of plan.workspace_bytes bytes. Returns (dq, dk, dv)."""
    fn = _load().bsm_attention_backward
    dev = plan.device
    refs = _refs(plan._q(q, "q"), plan._kv(k, "k"), plan._kv(v, "v"), plan._q(o, "o"),
                 plan._q(dout, "dout"), plan._q(dq, "dq"), plan._kv(dk, "dk"), plan._kv(dv, "dv"))
    lp = _contiguous(lse, torch.float32, plan.lse_elems, "lse", dev)
    wp, wn, workspace = _workspace(workspace, lambda: plan.workspace_bytes, dev, stream)
    _call(dev, fn, plan.handle, *refs[:4], lp, *refs[4:], _scale_of(scale, plan.head_dim), wp, wn,
          _stream(dev, stream))
    return dq, dk, dv


def _workspace(workspace, needed, index, stream):
    """(pointer, bytes, tensor) of the caller's workspace, or of one allocated for the call on the
    current stream."""
    if workspace is None:
        if stream is not None:
            raise ValueError("a call on a stream of its own needs its own workspace")
        workspace = torch.empty(needed(), dtype=torch.uint8, device=torch.device("cuda", index))
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{index}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


# ------------------------------------------------------------------------------ paged cache
def _cache_of(k_cache, v_cache) -> tuple[bsm_cache, int]:
    """k_cache, v_cache: bfloat16 tensors (pages, page size, heads, dim) of the same strides on one
    GPU, whose index is returned beside the cache."""
    shape, stride, index = k_cache.shape, k_cache.stride(), k_cache.get_device()
    if k_cache.dtype is not torch.bfloat16 or v_cache.dtype is not torch.bfloat16:
        raise TypeError(f"k_cache and v_cache must be bfloat16, got {k_cache.dtype} and {v_cache.dtype}")
    if index < 0 or v_cache.get_device() != index or len(shape) != 4:
        raise ValueError("k_cache and v_cache must be (pages, page size, heads, dim) on one GPU")
    if stride[3] != 1 and shape[3] > 1:
        raise ValueError("k_cache and v_cache: the last dimension must be contiguous")
    if shape != v_cache.shape or stride != v_cache.stride():
        raise ValueError("k_cache and v_cache must have the same shape and strides")
    return bsm_cache(k_cache.data_ptr(), v_cache.data_ptr(), shape[0], *stride[:3], *shape[1:],
                     0), index


def bsm_cache_slots(cached, fresh, page_size, n_pages, table, free_pages, n_free, q_start, kv_len,
                    slots, taken, stream=None):
    """Block table and slot map of a step from the requests' lengths (see bsm.h). int32 tensors on
    one GPU: cached, fresh, kv_len (batch), table (batch, width), free_pages, n_free (1),
    q_start (batch + 1), taken (2); slots: int64, as many as the step has room for tokens."""
    fn = _load().bsm_cache_slots
    batch, dev = cached.numel(), cached.get_device()
    if dev < 0:
        raise ValueError("cached must be a GPU tensor")
    if table.dim() != 2 or table.shape[0] < batch:
        raise ValueError(f"table of shape {tuple(table.shape)} has no row for each of {batch}")
    i32 = torch.int32
    _call(dev, fn, _contiguous(cached, i32, batch, "cached", dev),
          _contiguous(fresh, i32, batch, "fresh", dev), batch, *_int32(page_size=page_size),
          int(n_pages),
          _contiguous(table, i32, 0, "table", dev), table.shape[1],
          _contiguous(free_pages, i32, 0, "free_pages", dev), free_pages.numel(),
          _contiguous(n_free, i32, 1, "n_free", dev),
          _contiguous(q_start, i32, batch + 1, "q_start", dev),
          _contiguous(kv_len, i32, batch, "kv_len", dev),
          _contiguous(slots, torch.int64, 0, "slots", dev), slots.numel(),
          _contiguous(taken, i32, 2, "taken", dev), _stream(dev, stream))


def bsm_cache_append(k, v, slots, k_cache, v_cache, stream=None):
    """Writes the tokens of k and v (tokens, heads, dim) to their slots of the cache."""
    fn = _load().bsm_cache_append
    cache, dev = _cache_of(k_cache, v_cache)
    tokens = slots.numel()
    if k.dim() != 3 or v.dim() != 3:
        raise ValueError("k and v must be (tokens, heads, dim)")
    kr, vr = _refs(_operand(k, tokens, 1, cache.heads, cache.head_dim, "k", dev),
                   _operand(v, tokens, 1, cache.heads, cache.head_dim, "v", dev))
    _call(dev, fn, _ref(cache), kr, vr, _contiguous(slots, torch.int64, 0, "slots", dev), tokens,
          _stream(dev, stream))


def bsm_attention_paged_workspace(batch, tokens, heads_q, heads_kv, head_dim, max_q, max_kv,
                                  device=0) -> int:
    """Bytes of workspace that bsm_attention_paged needs for these sizes."""
    n = _i64()
    _check(_load().bsm_attention_paged_workspace(
        int(batch), int(tokens), *_int32(heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim,
                                         max_q=max_q, max_kv=max_kv, device=device), _ref(n)))
    return int(n.value)


def bsm_attention_paged(q, k_cache, v_cache, table, q_start, kv_len, o, max_q, max_kv=None,
                        window=0, scale=None, workspace=None, stream=None):
    """o = causal attention of every request's new tokens over its pages (see bsm.h). q, o:
    (tokens, heads, dim); table: int32 (batch, width); q_start: int32 (batch + 1); kv_len: int32
    (batch). max_q, max_kv: host bounds on a chunk and on kv_len (None or 0: the table's width).
    workspace: None (allocated for the call on the current stream; a call with a stream of its own
    brings its own) or a tensor of bsm_attention_paged_workspace bytes. Returns o."""
    fn = _load().bsm_attention_paged
    cache, dev = _cache_of(k_cache, v_cache)
    if q.dim() != 3 or o.dim() != 3:
        raise ValueError("q and o must be (tokens, heads, dim)")
    tokens, heads_q, _ = q.shape
    batch, dim = kv_len.numel(), cache.head_dim
    if table.dim() != 2 or table.shape[0] < batch:
        raise ValueError(f"table of shape {tuple(table.shape)} has no row for each of {batch}")
    qr, orr = _refs(_operand(q, tokens, 1, heads_q, dim, "q", dev),
                    _operand(o, tokens, 1, heads_q, dim, "o", dev))
    i32, width = torch.int32, table.shape[1]
    tp = _contiguous(table, i32, 0, "table", dev)
    sp = _contiguous(q_start, i32, batch + 1, "q_start", dev)
    lp = _contiguous(kv_len, i32, 0, "kv_len", dev)
    max_kv = width * cache.page_size if max_kv is None else int(max_kv) or width * cache.page_size
    max_q, max_kv, window = _int32(max_q=max_q, max_kv=max_kv, window=window)
    wp, wn, workspace = _workspace(
        workspace, lambda: bsm_attention_paged_workspace(batch, tokens, heads_q, cache.heads, dim,
                                                         max_q, max_kv, dev), dev, stream)
    _call(dev, fn, _ref(cache), qr, orr, tp, width, sp, lp, batch, tokens, heads_q, max_q, max_kv,
          window, _scale_of(scale, dim), wp, wn, _stream(dev, stream))
    return o
