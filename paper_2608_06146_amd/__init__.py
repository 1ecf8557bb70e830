"""PaDoc tree attention on MI355X: thin Python binding of ``libpadoc_attn``.

Every step of the computation runs in the HIP library; this module only
marshals arguments.  PyTorch provides device memory and the current stream; a
call's ``stream`` is where it runs instead (its inputs have to be ready there, its
results are read elsewhere after a wait).

    segs = segments_from_pages(pages, block_size=0)        # tree -> segments
    plan = TreePlan(segs, Hq, Hkv, d, "bf16", block_size=0,
                    num_kv_rows=T, num_q_rows=n_q)
    o, lse = tree_attn_fwd(q, k, v, plan)                    # packed forward
    o, lse = branch_decode(q, k_cache, v_cache, bt, plan)    # paged decode step

    rot = Rotary(d, "bf16", sections=(16, 24, 24))           # head norms and positions around it
    q, k = rotary_fwd(q, k, positions, rot, wq, wk)
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional, Sequence

import numpy as np

from . import _lib
from ._lib import PadocError, SEGMENT_DTYPE, WORK_DTYPE, RANGE_DTYPE, BWD_DTYPE

__all__ = ["TreePlan", "segments_from_pages", "segments_layout", "tree_attn_fwd", "tree_attn_bwd", "branch_decode",
           "DecodeSession", "tree_depths", "tree_remaining", "cache_from_rows", "Rotary", "rotary_fwd", "rotary_bwd",
           "rotary_append", "cache_copy_blocks", "PadocError", "SEGMENT_DTYPE", "version", "set_kernel_events", "make_workspace"]

_DTYPES = {"f32": _lib.F32, "fp32": _lib.F32, "float32": _lib.F32, "bf16": _lib.BF16, "bfloat16": _lib.BF16}


def version() -> str:
    return _lib.lib().padoc_version().decode()


def _page_struct(pg, keep):
    get = (lambda k: pg[k]) if isinstance(pg, dict) else (lambda k: getattr(pg, k))
    br = list(get("branches"))
    bget = lambda b, k: b[k] if isinstance(b, dict) else getattr(b, k)
    f = np.ascontiguousarray([bget(b, "fork") for b in br], dtype=np.int32)
    ln = np.ascontiguousarray([bget(b, "length") for b in br], dtype=np.int32)
    ql = np.ascontiguousarray([bget(b, "q_len") for b in br], dtype=np.int32)
    keep.extend([f, ln, ql])
    P = C.POINTER(C.c_int32)
    return _lib.Page(int(get("prefix_len")), int(get("prefix_q")), int(get("stream_len")), int(get("stream_q")),
                     len(br), f.ctypes.data_as(P), ln.ctypes.data_as(P), ql.ctypes.data_as(P))


def segments_from_pages(pages: Sequence, block_size: int = 0) -> np.ndarray:
    """Pages ``[prefix | stream | Y_1..Y_N]`` -> segment records in packed
    order (``padoc_tree_from_pages``)."""
    L = _lib.lib()
    keep: list = []
    arr = (_lib.Page * max(1, len(pages)))(*[_page_struct(p, keep) for p in pages])
    n = C.c_int32(0)
    L.padoc_tree_from_pages(arr, len(pages), block_size, None, 0, C.byref(n))
    out = np.zeros(n.value, dtype=SEGMENT_DTYPE)
    _lib.check(L.padoc_tree_from_pages(arr, len(pages), block_size, out.ctypes.data_as(C.c_void_p),
                                       n.value, C.byref(n)))
    return out


def segments_layout(nodes, block_size: int = 0) -> np.ndarray:
    """Generic nodes ``(parent, fork, len, q_len)`` -> segment records with the
    canonical packed offsets (``padoc_tree_layout``)."""
    out = np.zeros(len(nodes), dtype=SEGMENT_DTYPE)
    for i, n in enumerate(nodes):
        if isinstance(n, tuple):
            out[i] = (n[0], n[1], n[2], n[3], 0, 0)
        else:
            out[i] = (n.parent, n.fork, n.length, n.q_len, 0, 0)
    _lib.check(_lib.lib().padoc_tree_layout(out.ctypes.data_as(C.c_void_p), len(out), block_size))
    return out


def tree_depths(segments: np.ndarray):
    """Per page root of a segment tree: ``(root index, D_seq, D_crit)``
    arrays (``padoc_tree_depths``: sequential decoding depth and concurrent
    critical path, Sec. 3.1 / App. D); ``R_step = 1 - D_crit / D_seq``."""
    segs = np.ascontiguousarray(segments, dtype=SEGMENT_DTYPE)
    n = len(segs)
    d_seq = np.zeros(n, np.int64)
    d_crit = np.zeros(n, np.int64)
    _lib.check(_lib.lib().padoc_tree_depths(segs.ctypes.data if n else None, n, d_seq.ctypes.data,
                                            d_crit.ctypes.data))
    roots = np.nonzero(segs["parent"] < 0)[0]
    return roots, d_seq[roots], d_crit[roots]


def tree_remaining(segments: np.ndarray, progress=None) -> np.ndarray:
    """Remaining critical path of every segment (``padoc_tree_remaining``,
    Sec. 3.1) when segment s has produced ``progress[s]`` tokens (None: 0);
    int64, one entry per segment."""
    segs = np.ascontiguousarray(segments, dtype=SEGMENT_DTYPE)
    n = len(segs)
    prog = None
    if progress is not None:
        prog = np.ascontiguousarray(progress, dtype=np.int32)
        if prog.shape != (n,):
            raise ValueError(f"progress needs one entry per segment ({n}), got shape {prog.shape}")
    out = np.zeros(n, np.int64)
    _lib.check(_lib.lib().padoc_tree_remaining(segs.ctypes.data if n else None, n,
                                               prog.ctypes.data if prog is not None and n else None,
                                               out.ctypes.data if n else None))
    return out


def _on_stream(stream, device, call, *args):
    """``call(*args)`` on ``stream`` of GPU ``device``.  What it allocates comes
    from that stream's memory (a block that another stream let go of may still
    be in use by the work queued there); what it returns also belongs to the
    stream that was current, on which the caller reads it after a wait."""
    import torch
    if stream.device.index != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{device}")
    current = torch.cuda.current_stream(device)
    if device == torch._C._cuda_getDevice():  # torch.cuda.stream(stream), 3 us sooner
        torch.cuda.set_stream(stream)
        try:
            out = call(*args)
        finally:
            torch.cuda.set_stream(current)
    else:
        with torch.cuda.stream(stream):
            out = call(*args)
    for t in out if isinstance(out, tuple) else (out,):
        if t is not None and not any(t is a for a in args):
            t.record_stream(current)
    return out


def cache_from_rows(k_rows, v_rows, k_cache=None, v_cache=None, stream=None):
    """Paged K/V blocks in row layout ``[num_blocks, Hkv, 16, d]`` rewritten
    into the library's paged layouts (``padoc_cache_from_rows``): K
    ``[num_blocks, Hkv, d/8, 16, 8]``, V ``[num_blocks, Hkv, d, 16]``, block
    for block.  Returns ``(k_cache, v_cache)`` (allocated when not given)."""
    import torch
    if stream is not None and (k_cache is None or v_cache is None):
        return _on_stream(stream, k_rows.get_device(), cache_from_rows, k_rows, v_rows, k_cache, v_cache)
    if k_rows.dim() != 4 or k_rows.shape[2] != 16 or tuple(v_rows.shape) != tuple(k_rows.shape):
        raise ValueError("k_rows / v_rows must both be [num_blocks, Hkv, 16, d]")
    nb, hkv, _, d = k_rows.shape
    dt = k_rows.dtype
    if dt not in (torch.bfloat16, torch.float32) or v_rows.dtype != dt:
        raise ValueError("k_rows / v_rows must share dtype bfloat16 or float32")
    dev = k_rows.device
    for name, t in (("k_rows", k_rows), ("v_rows", v_rows)):
        _check_tensor(name, t, dt, dev)
    if k_cache is None:
        k_cache = torch.empty((nb, hkv, d // 8, 16, 8), dtype=dt, device=dev)
    if v_cache is None:
        v_cache = torch.empty((nb, hkv, d, 16), dtype=dt, device=dev)
    for name, t, shape in (("k_cache", k_cache, (nb, hkv, d // 8, 16, 8)), ("v_cache", v_cache, (nb, hkv, d, 16))):
        _check_tensor(name, t, dt, dev)
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {shape}")
    s = torch.cuda.current_stream(dev) if stream is None else stream
    _lib.check(_lib.lib().padoc_cache_from_rows(_ptr(k_rows), _ptr(v_rows), _ptr(k_cache), _ptr(v_cache), int(nb),
                                                int(hkv), int(d), _lib.BF16 if dt == torch.bfloat16 else _lib.F32,
                                                C.c_void_p(s.cuda_stream)))
    return k_cache, v_cache


class TreePlan:
    """A validated tree and its schedule (``padoc_plan``)."""

    def __init__(self, segments: np.ndarray, num_heads_q: int, num_heads_kv: int, head_dim: int,
                 dtype: str = "bf16", block_size: int = 0, num_kv_rows: int = 0, num_q_rows: Optional[int] = None,
                 softmax_scale: Optional[float] = None, block_table_host: Optional[np.ndarray] = None,
                 block_table_len: Optional[int] = None, max_chunk_keys: int = 0, target_workgroups: int = 0):
        segs = np.ascontiguousarray(segments, dtype=SEGMENT_DTYPE)
        self.segments = segs
        self.num_heads_q, self.num_heads_kv, self.head_dim = num_heads_q, num_heads_kv, head_dim
        self.dtype = dtype
        self.block_size = block_size
        if num_q_rows is None:
            num_q_rows = int((segs["q_off"] + segs["q_len"]).max()) if len(segs) else 0
        self.num_q_rows = num_q_rows
        self.softmax_scale = 1.0 / math.sqrt(head_dim) if softmax_scale is None else softmax_scale
        bt = None
        if block_table_host is not None:
            bt = np.ascontiguousarray(block_table_host, dtype=np.int32)
            if block_table_len is None:
                block_table_len = bt.size
        if block_table_len is None:
            block_table_len = 0
        self.block_table_len = block_table_len
        desc = _lib.TreeDesc(len(segs), segs.ctypes.data if len(segs) else None, num_heads_q, num_heads_kv,
                             head_dim, float(self.softmax_scale), _DTYPES[dtype], block_size, int(num_kv_rows),
                             int(num_q_rows), bt.ctypes.data if bt is not None else None, int(block_table_len),
                             int(max_chunk_keys), int(target_workgroups))
        h = C.c_void_p()
        L = _lib.lib()
        _lib.check(L.padoc_plan_create(C.byref(desc), C.byref(h)))
        self._h = h
        sz = C.c_size_t(0)
        _lib.check(L.padoc_plan_workspace_bytes(h, C.byref(sz)))
        self.workspace_bytes = sz.value
        self._ws = None

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("plan is closed")
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None:
            _lib.lib().padoc_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def export(self) -> dict:
        """Schedule as numpy arrays (copies)."""
        return _export_schedule(self.handle)

    def backward_workspace_bytes(self) -> int:
        n = C.c_size_t(0)
        _lib.check(_lib.lib().padoc_plan_backward_workspace_bytes(self.handle, C.byref(n)))
        return int(n.value)

    def backward_workspace(self, device):
        """A cached device workspace for the backward (256-byte aligned)."""
        self._bws = _workspace(getattr(self, "_bws", None), self.backward_workspace_bytes(), device)
        return self._bws[2]

    def workspace(self, device):
        """A cached device workspace of the plan's size (256-byte aligned)."""
        self._ws = _workspace(self._ws, self.workspace_bytes, device)
        return self._ws[2]


def _workspace(held, nbytes, device):
    """``(device, allocation, workspace, streams)``: ``held`` where it is on
    ``device``, else a new one.  It belongs to the streams that were current when
    it was asked for: a plan may go while work is queued on any of them."""
    import torch
    dev = torch.device(device)
    if held is None or held[0] != dev:
        raw = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
        off = (-raw.data_ptr()) % 256
        held = (dev, raw, raw[off: off + nbytes], set())
    s = torch._C._cuda_getCurrentRawStream(held[1].get_device()) if held[1].is_cuda else None
    if s is not None and s not in held[3]:
        held[1].record_stream(torch.cuda.current_stream(dev))  # (nothing, on the stream it was allocated on)
        held[3].add(s)
    return held


def _carray(ptr, n, dt):
    if n == 0 or not ptr:
        return np.zeros(0, dtype=dt)
    buf = (C.c_char * (int(n) * np.dtype(dt).itemsize)).from_address(ptr)
    return np.frombuffer(buf, dtype=dt).copy()


def _export_schedule(handle) -> dict:
    v = _lib.ScheduleView()
    _lib.check(_lib.lib().padoc_plan_export(handle, C.byref(v)))
    arr = _carray
    return {
        "kind": v.kind, "tile_cols": v.tile_cols, "tile_keys": v.tile_keys, "n_work_shared": v.n_work_shared,
        "work": arr(v.work, v.n_work, WORK_DTYPE), "ranges": arr(v.ranges, v.n_range, RANGE_DTYPE),
        "lims": arr(v.lims, v.n_lim, np.int32), "toks": arr(v.toks, v.n_tok, np.int32),
        "tile_class": arr(v.tile_class, v.n_tile_class, np.int8),
        "tile_class_off": arr(v.tile_class_off, v.n_range, np.int64),
        "comb_ptr": arr(v.comb_ptr, v.n_comb_ptr, np.int32), "comb_slot": arr(v.comb_slot, v.n_comb, np.int32),
        "comb_rows": arr(v.comb_rows, v.n_comb_rows, np.int32),
        "bwd": arr(v.bwd, v.n_bwd, BWD_DTYPE), "btoks": arr(v.btoks, v.n_btok, np.int32),
        "blims": arr(v.blims, v.n_blim, np.int32),
        "n_slots": v.n_slots, "workspace_bytes": v.workspace_bytes,
    }


def make_workspace(plan: TreePlan, device):
    return plan.workspace(device)


def _ptr(t):
    return C.c_void_p(t.data_ptr())


def _check_tensor(name, t, dtype, device):
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _torch_dtype(plan):
    import torch
    return torch.bfloat16 if _DTYPES[plan.dtype] == _lib.BF16 else torch.float32


def _outputs(plan, q, out, lse):
    import torch
    if out is None:
        out = torch.empty(plan.num_q_rows, plan.num_heads_q, plan.head_dim, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(plan.num_q_rows, plan.num_heads_q, dtype=torch.float32, device=q.device)
    return out, lse


def tree_attn_fwd(q, k, v, plan: TreePlan, out=None, lse=None, workspace=None, stream=None):
    """Packed forward (``padoc_tree_attn_fwd``).  q ``[n_q, Hq, d]``; k, v
    ``[T, Hkv, d]``; returns ``(O [n_q, Hq, d], LSE [n_q, Hq] float32)``."""
    import torch
    if stream is not None and any(t is None for t in (out, lse, workspace)):
        return _on_stream(stream, q.get_device(), tree_attn_fwd, q, k, v, plan, out, lse, workspace)
    dt = _torch_dtype(plan)
    dev = q.device
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_tensor(name, t, dt, dev)
    out, lse = _outputs(plan, q, out, lse)
    ws = plan.workspace(dev) if workspace is None else workspace
    s = torch.cuda.current_stream(dev) if stream is None else stream
    _lib.check(_lib.lib().padoc_tree_attn_fwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
                                              _ptr(ws), ws.numel(), C.c_void_p(s.cuda_stream)))
    return out, lse


def _repeat_call(plan, key):
    """The C arguments of the plan's previous call when this call passes the
    same tensors (same objects at the same addresses) on the same stream,
    else None.  A decode loop calls with the same buffers every step; this
    skips the per-call checks and argument marshalling."""
    last = getattr(plan, "_last_call", None)
    return last[1] if last is not None and last[0] == key else None


def branch_decode(q, k_cache, v_cache, block_table, plan: TreePlan, out=None, lse=None, workspace=None,
                  stream=None):
    """Decode step over a paged cache (``padoc_branch_decode``).  q ``[n_q,
    Hq, d]``; K cache chunk-major ``[blocks, Hkv, d/8, 16, 8]``, V cache
    d-major ``[blocks, Hkv, d, 16]`` (layouts in ``padoc_attn.h``);
    block_table int32 on the device; returns ``(O, LSE)``."""
    import torch
    if out is not None and lse is not None and workspace is not None:
        s = torch.cuda.current_stream(q.device) if stream is None else stream
        key = ("decode", plan.handle, s.cuda_stream) + tuple(
            (id(t), t.data_ptr(), t.shape, t.stride(), t.dtype) for t in (q, k_cache, v_cache, block_table, out, lse, workspace))
        args = _repeat_call(plan, key)
        if args is not None:
            _lib.check(_lib.lib().padoc_branch_decode(*args))
            return out, lse
    elif stream is not None:
        return _on_stream(stream, q.get_device(), branch_decode, q, k_cache, v_cache, block_table, plan, out, lse, workspace)
    dt = _torch_dtype(plan)
    dev = q.device
    for name, t in (("q", q), ("k_cache", k_cache), ("v_cache", v_cache)):
        _check_tensor(name, t, dt, dev)
    _check_tensor("block_table", block_table, torch.int32, dev)
    out, lse = _outputs(plan, q, out, lse)
    ws = plan.workspace(dev) if workspace is None else workspace
    s = torch.cuda.current_stream(dev) if stream is None else stream
    args = (plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(out), _ptr(lse), _ptr(ws),
            ws.numel(), C.c_void_p(s.cuda_stream))
    _lib.check(_lib.lib().padoc_branch_decode(*args))
    if workspace is not None:
        plan._last_call = (("decode", plan.handle, s.cuda_stream) + tuple(
            (id(t), t.data_ptr(), t.shape, t.stride(), t.dtype) for t in (q, k_cache, v_cache, block_table, out, lse, workspace)),
            args)
    return out, lse


NO_ALLOC_WORKSPACE_BYTES = 64 << 20   # PADOC_NO_ALLOC_WORKSPACE_BYTES


def plan_upload(plan: TreePlan, workspace, stream=None):
    """Copy a decode plan's schedule into ``workspace`` (``padoc_plan_upload``)
    for ``branch_decode_resident`` calls: every layer of a decode step runs
    over the same tree, so one upload serves all of them."""
    import torch
    _check_tensor("workspace", workspace, torch.uint8, workspace.device)
    s = torch.cuda.current_stream(workspace.device) if stream is None else stream
    _lib.check(_lib.lib().padoc_plan_upload(plan.handle, _ptr(workspace), workspace.numel(),
                                            C.c_void_p(s.cuda_stream)))
    return workspace


def branch_decode_resident(q, k_cache, v_cache, block_table, plan: TreePlan, out, lse, workspace, stream=None):
    """Decode step on a workspace that holds the plan's schedule
    (``padoc_branch_decode_resident``, after ``plan_upload``): the kernels of
    ``branch_decode`` without the schedule copy."""
    import torch
    s = torch.cuda.current_stream(q.device) if stream is None else stream
    key = ("resident", plan.handle, s.cuda_stream) + tuple(
        (id(t), t.data_ptr(), t.shape, t.stride(), t.dtype) for t in (q, k_cache, v_cache, block_table, out, lse, workspace))
    args = _repeat_call(plan, key)
    if args is None:
        dt = _torch_dtype(plan)
        dev = q.device
        for name, t in (("q", q), ("k_cache", k_cache), ("v_cache", v_cache), ("out", out)):
            _check_tensor(name, t, dt, dev)
        _check_tensor("block_table", block_table, torch.int32, dev)
        _check_tensor("lse", lse, torch.float32, dev)
        _check_tensor("workspace", workspace, torch.uint8, dev)
        args = (plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(out), _ptr(lse),
                _ptr(workspace), workspace.numel(), C.c_void_p(s.cuda_stream))
    _lib.check(_lib.lib().padoc_branch_decode_resident(*args))
    plan._last_call = (key, args)
    return out, lse


def branch_decode_no_alloc(q, k_cache, v_cache, block_table, plan: TreePlan, out, lse, stream=None):
    """Decode step with the library's fixed per-GPU workspace
    (``padoc_branch_decode_no_alloc``): the caller passes every input and
    both outputs; nothing is allocated.  Calls that overlap on one GPU race
    on that workspace."""
    import torch
    dt = _torch_dtype(plan)
    dev = q.device
    for name, t in (("q", q), ("k_cache", k_cache), ("v_cache", v_cache), ("out", out)):
        _check_tensor(name, t, dt, dev)
    _check_tensor("block_table", block_table, torch.int32, dev)
    _check_tensor("lse", lse, torch.float32, dev)
    s = torch.cuda.current_stream(dev) if stream is None else stream
    _lib.check(_lib.lib().padoc_branch_decode_no_alloc(plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                                       _ptr(block_table), _ptr(out), _ptr(lse),
                                                       C.c_void_p(s.cuda_stream)))
    return out, lse


def tree_attn_bwd(q, k, v, o, lse, dout, plan: TreePlan, dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Backward of the packed forward (``padoc_tree_attn_bwd``, bf16 plans).
    q, o, dout ``[n_q, Hq, d]``; k, v ``[T, Hkv, d]``; lse float32 ``[n_q,
    Hq]`` (the forward's outputs); returns ``(dQ, dK, dV)``."""
    import torch
    if stream is not None and any(t is None for t in (dq, dk, dv, workspace)):
        return _on_stream(stream, q.get_device(), tree_attn_bwd, q, k, v, o, lse, dout, plan, dq, dk, dv, workspace)
    dt = _torch_dtype(plan)
    dev = q.device
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o), ("dout", dout)):
        _check_tensor(name, t, dt, dev)
    _check_tensor("lse", lse, torch.float32, dev)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    for name, t, ref in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        _check_tensor(name, t, dt, dev)
        if t.shape != ref.shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(ref.shape)}")
    ws = plan.backward_workspace(dev) if workspace is None else workspace
    s = torch.cuda.current_stream(dev) if stream is None else stream
    _lib.check(_lib.lib().padoc_tree_attn_bwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dout),
                                              _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), ws.numel(),
                                              C.c_void_p(s.cuda_stream)))
    return dq, dk, dv


_STYLES = {"halves": 0, "pairs": 1}  # padoc_rotary_style


class Rotary:
    """Head norms and rotary positions of a decoder layer (``padoc_rotary``):
    the first ``rotary_dim`` dimensions (default: all) of every head are
    rotated by the positions of up to four axes.  ``axis[i]`` is the axis of
    pair i (of ``n_axes``; default: as many as it names), or ``sections`` counts
    the pairs of each axis in order; neither: one axis.  ``inv_freq`` (radians per position of each pair) replaces
    ``base ** (-2 i / rotary_dim)``.  ``style``: "halves" pairs dimensions i
    and i + rotary_dim/2, "pairs" 2i and 2i + 1.  ``scale`` multiplies the
    cosines and sines; ``eps`` belongs to the norms (used where a call passes
    weights).  Host memory only."""

    def __init__(self, head_dim: int, dtype: str = "bf16", rotary_dim: Optional[int] = None, sections=None, axis=None,
                 base: float = 10000.0, inv_freq=None, style: str = "halves", scale: float = 1.0, eps: float = 1e-6,
                 n_axes: Optional[int] = None):
        self.head_dim, self.dtype = int(head_dim), dtype
        self.rotary_dim = self.head_dim if rotary_dim is None else int(rotary_dim)
        if style not in _STYLES:
            raise ValueError(f"style {style!r} is not one of {sorted(_STYLES)}")
        if sections is not None:
            if axis is not None:
                raise ValueError("pass sections or axis, not both")
            axis = np.repeat(np.arange(len(sections)), sections)
        pairs = self.rotary_dim // 2
        ax = None if axis is None else np.ascontiguousarray(axis, dtype=np.int32)
        fr = None if inv_freq is None else np.ascontiguousarray(inv_freq, dtype=np.float64)
        for name, a in (("axis / sections", ax), ("inv_freq", fr)):
            if a is not None and a.shape != (pairs,):
                raise ValueError(f"{name} must cover the {pairs} rotated pairs, got shape {a.shape}")
        if n_axes is None:
            n_axes = 1 if ax is None else len(sections) if sections is not None else int(ax.max(initial=0)) + 1
        self.n_axes = int(n_axes)
        desc = _lib.RotaryDesc(self.head_dim, self.rotary_dim, self.n_axes, _STYLES[style],
                               ax.ctypes.data if ax is not None else None,
                               fr.ctypes.data if fr is not None else None, float(base), float(scale), float(eps),
                               _DTYPES[dtype])
        h = C.c_void_p()
        _lib.check(_lib.lib().padoc_rotary_create(C.byref(desc), C.byref(h)))
        self._h = h
        self.torch_dtype = _torch_dtype(self)
        self._rows = _lib.rows(h, self.head_dim, self.n_axes, _DTYPES[dtype] == _lib.BF16)

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("rotary is closed")
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None:
            self._rows = None
            _lib.lib().padoc_rotary_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_NO_HEADS = (0, 0, 0)


def _heads(name, t, dt, device, shape):
    """``(data, row stride, head stride)`` of rows of heads ``[n, H, d]`` on
    GPU ``device``."""
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{device}")
    if t.dtype is not dt:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dt}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    rs, hs, es = t.stride()
    if es != 1:
        raise ValueError(f"{name}: the head dimension must be contiguous")
    return t.data_ptr(), rs, hs


def _rows_of(rotary, like):
    """GPU index and dtype of the rows of a call, by one of their tensors."""
    import torch
    if not isinstance(like, torch.Tensor):
        raise TypeError("rows must be torch tensors")
    device, dt = like.get_device(), rotary.torch_dtype
    if device < 0:
        raise ValueError(f"rows are on {like.device}, expected a GPU")
    if like.dtype is not dt:
        raise TypeError(f"rows have dtype {like.dtype}, the rotary is for {rotary.dtype}")
    if like.dim() != 3 or like.shape[2] != rotary.head_dim:
        raise ValueError(f"rows must be [n, H, {rotary.head_dim}], got {tuple(like.shape)}")
    return device, dt


def _weight(name, w, dt, device, d):
    """Address of a norm's weight ``[d]``, 0 for None."""
    if w is None:
        return 0
    if w.dtype is not dt or w.get_device() != device or not w.is_contiguous():
        import torch
        _check_tensor(name, w, dt, torch.device("cuda", device))
    if w.shape != (d,):
        raise ValueError(f"{name} has shape {tuple(w.shape)}, expected {(d,)}")
    return w.data_ptr()


def _positions(name, pos, rotary, n, device):
    """``(address, axis stride)`` of int32 positions ``[n_axes, n]`` (``[n]``
    for one axis)."""
    import torch
    if pos.get_device() != device:
        raise ValueError(f"{name} is on {pos.device}, expected cuda:{device}")
    if pos.dtype is not torch.int32:
        raise TypeError(f"{name} has dtype {pos.dtype}, expected torch.int32")
    axes = rotary.n_axes
    if axes == 1 and pos.dim() == 1:
        pos = pos[None]
    if pos.shape != (axes, n):
        raise ValueError(f"{name} has shape {tuple(pos.shape)}, expected {(axes, n)}")
    rs, es = pos.stride()
    if n > 1 and es != 1:
        raise ValueError(f"{name}: the positions of an axis must be contiguous")
    return pos.data_ptr(), rs if axes > 1 else 0


def _launch(f, device, *args):
    """``f(*args, stream)`` on GPU ``device`` and its current stream."""
    import torch
    s = torch._C._cuda_getCurrentRawStream(device)  # current_stream().cuda_stream, 1.7 us sooner
    if device == torch._C._cuda_getDevice():
        _lib.check(f(*args, s))
    else:
        with torch.cuda.device(device):
            _lib.check(f(*args, s))


def rotary_fwd(q, k, positions, rotary: Rotary, q_weight=None, k_weight=None, q_out=None, k_out=None, stream=None):
    """Per-head RMS norm (where weights ``[d]`` are given) and rotation of q
    ``[n, Hq, d]`` and k ``[n, Hkv, d]`` by ``positions`` (int32 ``[n_axes,
    n]``; ``padoc_rotary_fwd``).  Rows and heads may be strided, as in slices
    of a fused projection; q or k may be None, and q_out / k_out may be q / k.
    Returns ``(q_out, k_out)``."""
    if stream is not None:
        return _on_stream(stream, _rows_of(rotary, k if q is None else q)[0], rotary_fwd, q, k, positions, rotary, q_weight,
                          k_weight, q_out, k_out)
    if rotary._rows is not None:
        done = rotary._rows.fwd(q, k, positions, q_weight, k_weight, q_out, k_out)
        if done is not None:
            return done if type(done) is tuple else _lib.check(done)
    like = k if q is None else q
    device, dt = _rows_of(rotary, like)
    n, d = like.shape[0], rotary.head_dim
    hq = hk = 0
    q_in = q_to = k_in = k_to = _NO_HEADS
    if q is not None:
        hq = q.shape[1]
        shape = (n, hq, d)
        q_in = _heads("q", q, dt, device, shape)
        if q_out is None:
            q_out = q.new_empty(shape)
            q_to = q_out.data_ptr(), hq * d, d
        else:
            q_to = _heads("q_out", q_out, dt, device, shape)
    if k is not None:
        hk = k.shape[1] if k.dim() == 3 else 0
        shape = (n, hk, d)
        k_in = _heads("k", k, dt, device, shape)
        if k_out is None:
            k_out = k.new_empty(shape)
            k_to = k_out.data_ptr(), hk * d, d
        else:
            k_to = _heads("k_out", k_out, dt, device, shape)
    args = _lib.ROTARY_FWD_ARGS.pack(n, hq, hk, *_positions("positions", positions, rotary, n, device), *q_in, *k_in,
                                     *q_to, *k_to, _weight("q_weight", q_weight, dt, device, d),
                                     _weight("k_weight", k_weight, dt, device, d))
    _launch(_lib.lib().padoc_rotary_fwd, device, rotary.handle, args)
    return (None if q is None else q_out), (None if k is None else k_out)


def rotary_bwd(dq_out, dk_out, positions, rotary: Rotary, q=None, k=None, q_weight=None, k_weight=None, dq=None,
               dk=None, weight_grads: bool = True, stream=None):
    """Gradients of ``rotary_fwd`` (``padoc_rotary_bwd``): dq_out / dk_out are
    those of its outputs, q / k its inputs (read only where there is a
    weight).  Returns ``(dq, dk, dq_weight, dk_weight)``; the weights'
    gradients are float32 ``[d]``, None without a weight or with
    ``weight_grads=False``."""
    if stream is not None:
        return _on_stream(stream, _rows_of(rotary, dk_out if dq_out is None else dq_out)[0], rotary_bwd, dq_out, dk_out,
                          positions, rotary, q, k, q_weight, k_weight, dq, dk, weight_grads)
    if rotary._rows is not None:
        done = rotary._rows.bwd(dq_out, dk_out, positions, q, k, q_weight, k_weight, dq, dk, weight_grads)
        if done is not None:
            return done if type(done) is tuple else _lib.check(done)
    import torch
    like = dk_out if dq_out is None else dq_out
    device, dt = _rows_of(rotary, like)
    n, d = like.shape[0], rotary.head_dim
    heads, counts, outs, ws, dws = [], [], [], [], []
    for name, g, x, w, out in (("q", dq_out, q, q_weight, dq), ("k", dk_out, k, k_weight, dk)):
        if g is None:
            heads.append((_NO_HEADS,) * 3), counts.append(0), outs.append(None), ws.append(0), dws.append(None)
            continue
        h = g.shape[1] if g.dim() == 3 else 0
        shape = (n, h, d)
        g_in, x_in = _heads(f"d{name}_out", g, dt, device, shape), _NO_HEADS
        if w is not None:
            if x is None:
                raise ValueError(f"the backward of {name}'s norm needs {name}")
            x_in = _heads(name, x, dt, device, shape)
        if out is None:
            out = g.new_empty(shape)
            to = out.data_ptr(), h * d, d
        else:
            to = _heads("d" + name, out, dt, device, shape)
        heads.append((x_in, g_in, to)), counts.append(h), outs.append(out)
        ws.append(_weight(name + "_weight", w, dt, device, d))
        dws.append(g.new_empty(d, dtype=torch.float32) if w is not None and weight_grads else None)
    hq, hk = counts
    L, handle = _lib.lib(), rotary.handle
    wptr, wbytes = None, 0
    if dws[0] is not None or dws[1] is not None:
        nb = C.c_size_t(0)
        _lib.check(L.padoc_rotary_bwd_workspace_bytes(handle, n, hq, hk, C.byref(nb)))
        work = like.new_empty(nb.value, dtype=torch.uint8)  # the allocator's blocks are 512-byte aligned
        wptr, wbytes = work.data_ptr(), nb.value
    (xq, gq, oq), (xk, gk, ok) = heads
    args = _lib.ROTARY_BWD_ARGS.pack(n, hq, hk, *_positions("positions", positions, rotary, n, device), *xq, *xk, *gq,
                                     *gk, *oq, *ok, *ws, *(0 if t is None else t.data_ptr() for t in dws))
    _launch(L.padoc_rotary_bwd, device, handle, args, wptr, wbytes)
    return outs[0], outs[1], dws[0], dws[1]


def _append_args(rotary, q, k, v, positions, q_weight, k_weight, q_positions, q_out, slots=0, k_cache=0, v_cache=0,
                 num_blocks=0):
    """The packed arguments of an append, its q_out and the GPU's index."""
    device, dt = _rows_of(rotary, q if k is None else k)
    d = rotary.head_dim
    n_q = hq = n = hk = 0
    q_in = q_to = k_in = v_in = _NO_HEADS
    q_pos = pos = (0, 0)
    if k is not None:
        n, hk, _ = shape = k.shape
        k_in, v_in = _heads("k", k, dt, device, shape), _heads("v", v, dt, device, shape)
        pos = _positions("positions", positions, rotary, n, device)
    if q is not None:
        if q.dim() != 3:
            raise ValueError(f"q has shape {tuple(q.shape)}, expected [n, H, {d}]")
        n_q, hq, _ = q.shape
        shape = (n_q, hq, d)
        q_in = _heads("q", q, dt, device, shape)
        if q_out is None:
            q_out = q.new_empty(shape)
            q_to = q_out.data_ptr(), hq * d, d
        else:
            q_to = _heads("q_out", q_out, dt, device, shape)
        if q_positions is not None:
            q_pos = _positions("q_positions", q_positions, rotary, n_q, device)
        elif k is None:
            q_pos = _positions("positions", positions, rotary, n_q, device)
    args = _lib.ROTARY_APPEND_ARGS.pack(n_q, n, hq, hk, *q_pos, *pos, *q_in, *k_in, *v_in, *q_to,
                                        _weight("q_weight", q_weight, dt, device, d),
                                        _weight("k_weight", k_weight, dt, device, d), slots, k_cache, v_cache, num_blocks)
    return args, None if q is None else q_out, device


def _check_caches(k_cache, v_cache, dtype, dev):
    """Checks caches in the library's layouts; ``(blocks, Hkv, d)``."""
    _check_tensor("k_cache", k_cache, dtype, dev)
    _check_tensor("v_cache", v_cache, dtype, dev)
    nb, hkv, d, slots = v_cache.shape if v_cache.dim() == 4 else (0, 0, 0, 0)
    if slots != 16 or k_cache.shape != (nb, hkv, d // 8, 16, 8):
        raise ValueError(f"caches must be K [blocks, Hkv, d/8, 16, 8] and V [blocks, Hkv, d, 16], got "
                         f"{tuple(k_cache.shape)} and {tuple(v_cache.shape)}")
    return nb, hkv, d


def rotary_append(q, k, v, positions, slots, k_cache, v_cache, rotary: Rotary, q_weight=None, k_weight=None,
                  q_positions=None, q_out=None, stream=None):
    """A decode step's rows (``padoc_rotary_append``): q ``[n_q, Hq, d]``
    normed and rotated into ``q_out``, k and v ``[n_new, Hkv, d]`` into the
    caches (k normed and rotated) at ``slots`` (int32 ``[n_new, 2]``: block id
    and slot; a block id of -1 leaves the row out).  ``q_positions`` may be
    left out when query row i is new row i; q may be None.  Returns q_out."""
    if stream is not None:
        return _on_stream(stream, _rows_of(rotary, q if k is None else k)[0], rotary_append, q, k, v, positions, slots,
                          k_cache, v_cache, rotary, q_weight, k_weight, q_positions, q_out)
    if rotary._rows is not None:
        done = rotary._rows.append(q, k, v, positions, slots, k_cache, v_cache, q_weight, k_weight, q_positions, q_out)
        if done is not None:
            return done[0] if type(done) is tuple else _lib.check(done)
    import torch
    if k is None or v is None:
        raise ValueError("rotary_append needs k and v (rotary_fwd rotates q alone)")
    dev = k.device
    nb, hkv, d = _check_caches(k_cache, v_cache, rotary.torch_dtype, dev)
    if k.shape[1:] != (hkv, d) or d != rotary.head_dim:
        raise ValueError(f"the caches hold {hkv} heads of {d}, the rows are {tuple(k.shape)}")
    _check_tensor("slots", slots, torch.int32, dev)
    if slots.shape != (k.shape[0], 2):
        raise ValueError(f"slots has shape {tuple(slots.shape)}, expected {(k.shape[0], 2)}")
    args, q_out, device = _append_args(rotary, q, k, v, positions, q_weight, k_weight, q_positions, q_out,
                                       slots.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), nb)
    _launch(_lib.lib().padoc_rotary_append, device, rotary.handle, args)
    return q_out


def _copy_blocks(k_cache, v_cache, pairs):
    """The native call; its first use finds it."""
    global _copy_blocks
    _copy_blocks = _lib.native_copy_blocks()
    return _copy_blocks(k_cache, v_cache, pairs)


def cache_copy_blocks(k_cache, v_cache, pairs, k_dst=None, v_dst=None, pairs_host=None, stream=None):
    """Copy blocks ``pairs[i, 0]`` of the paged caches to blocks ``pairs[i,
    1]`` of the same caches, or of ``k_dst`` / ``v_dst``
    (``padoc_cache_copy_blocks``; int32 ``[n, 2]`` on the device, with an
    optional host copy that is only checked).  Returns the caches written."""
    if stream is not None:
        if not k_cache.is_cuda:
            raise ValueError(f"k_cache is on {k_cache.device}, expected a GPU")
        return _on_stream(stream, k_cache.get_device(), cache_copy_blocks, k_cache, v_cache, pairs, k_dst, v_dst, pairs_host)
    if k_dst is None and v_dst is None and pairs_host is None:
        done = _copy_blocks(k_cache, v_cache, pairs)
        if done is not None:
            if done:
                _lib.check(done)
            return k_cache, v_cache
    import torch
    if (k_dst is None) != (v_dst is None):
        raise ValueError("pass k_dst and v_dst together (or neither)")
    dev, dt = k_cache.device, k_cache.dtype
    if not k_cache.is_cuda:
        raise ValueError(f"k_cache is on {dev}, expected a GPU")
    if dt not in (torch.bfloat16, torch.float32):
        raise TypeError(f"caches must be bfloat16 or float32, got {dt}")
    nb, hkv, d = _check_caches(k_cache, v_cache, dt, dev)
    if k_dst is None:
        k_dst, v_dst, nd = k_cache, v_cache, nb
    else:
        nd, h2, d2 = _check_caches(k_dst, v_dst, dt, dev)
        if (h2, d2) != (hkv, d):
            raise ValueError(f"blocks of {hkv} heads of {d} do not fit caches of {h2} heads of {d2}")
    _check_tensor("pairs", pairs, torch.int32, dev)
    if pairs.dim() != 2 or pairs.shape[1] != 2:
        raise ValueError(f"pairs has shape {tuple(pairs.shape)}, expected [n, 2]")
    host = None
    if pairs_host is not None:
        host = np.ascontiguousarray(pairs_host, dtype=np.int32)
        if host.shape != pairs.shape:
            raise ValueError(f"pairs_host has shape {host.shape}, expected {tuple(pairs.shape)}")
    _launch(_lib.lib().padoc_cache_copy_blocks, dev.index, k_cache.data_ptr(), v_cache.data_ptr(), nb,
            k_dst.data_ptr(), v_dst.data_ptr(), nd, pairs.data_ptr(), pairs.shape[0],
            None if host is None else host.ctypes.data, hkv, d, _lib.BF16 if dt == torch.bfloat16 else _lib.F32)
    return k_dst, v_dst


class DecodeSession:
    """Decode session (``padoc_session_*``): the step loop of masked parallel
    decoding (App. E) over caller-owned paged caches.

    ``open(parent, fork)`` starts a stream (``parent=-1``: a page root) that
    sees the first ``fork`` tokens of ``parent``; ``close(id)`` retires one.
    A step is ``prepare(n_new, n_query)`` (host: grow every open stream by
    ``n_new[i]`` tokens, plan the attention of the last ``n_query[i]``) then
    ``launch(q, k_new, v_new)`` (device: append the K/V rows, patch the block
    table, attention); rows follow ascending open stream id.  Without caches
    (``k_cache=None``) the session is host-only: steps are completed with
    ``commit()`` and inspected with ``view()``."""

    def __init__(self, num_heads_q: int, num_heads_kv: int, head_dim: int, num_blocks: int, dtype: str = "bf16",
                 k_cache=None, v_cache=None, block_table=None, block_table_capacity: Optional[int] = None,
                 softmax_scale: Optional[float] = None, max_chunk_keys: int = 0, target_workgroups: int = 0):
        self.num_heads_q, self.num_heads_kv, self.head_dim = num_heads_q, num_heads_kv, head_dim
        self.dtype = dtype
        self.num_blocks = int(num_blocks)
        self.softmax_scale = 1.0 / math.sqrt(head_dim) if softmax_scale is None else softmax_scale
        dev = (k_cache, v_cache, block_table)
        if any(t is not None for t in dev) and any(t is None for t in dev):
            raise ValueError("pass k_cache, v_cache and block_table together (or none of them)")
        self.k_cache, self.v_cache, self.block_table = k_cache, v_cache, block_table
        if block_table is not None:
            import torch
            dt = torch.bfloat16 if _DTYPES[dtype] == _lib.BF16 else torch.float32
            dv = k_cache.device
            _check_tensor("k_cache", k_cache, dt, dv)
            _check_tensor("v_cache", v_cache, dt, dv)
            _check_tensor("block_table", block_table, torch.int32, dv)
            want_k = (self.num_blocks, num_heads_kv, head_dim // 8, 16, 8)
            want_v = (self.num_blocks, num_heads_kv, head_dim, 16)
            if tuple(k_cache.shape) != want_k or tuple(v_cache.shape) != want_v:
                raise ValueError(f"caches must be K {want_k} and V {want_v}")
            if block_table_capacity is None:
                block_table_capacity = block_table.numel()
            if block_table_capacity > block_table.numel():
                raise ValueError("block_table_capacity exceeds the block table")
            self.device = dv
        else:
            self.device = None
        if block_table_capacity is None:
            block_table_capacity = 2 * self.num_blocks + 1024
        self.block_table_capacity = int(block_table_capacity)
        desc = _lib.SessionDesc(num_heads_q, num_heads_kv, head_dim, float(self.softmax_scale), _DTYPES[dtype],
                                self.num_blocks, self.block_table_capacity,
                                k_cache.data_ptr() if k_cache is not None else None,
                                v_cache.data_ptr() if v_cache is not None else None,
                                block_table.data_ptr() if block_table is not None else None,
                                int(max_chunk_keys), int(target_workgroups))
        h = C.c_void_p()
        _lib.check(_lib.lib().padoc_session_create(C.byref(desc), C.byref(h)))
        self._h = h
        self._streams = _lib.streams(h)
        self.n_open = 0
        self.n_kv_rows = self.n_q_rows = 0
        self.workspace_bytes = 0
        self._ws = None
        self._users = set()  # streams of _keep

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("session is closed")
        return self._h

    def destroy(self):
        if getattr(self, "_h", None) is not None:
            _lib.lib().padoc_session_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def open(self, parent: int = -1, fork: int = 0) -> int:
        if self._h is None:
            raise ValueError("session is closed")
        i = self._streams.open(parent, fork)
        if i < 0:
            _lib.check(i)
        self.n_open += 1
        return i

    def close(self, stream_id: int) -> None:
        if self._h is None:
            raise ValueError("session is closed")
        st = self._streams.close(stream_id)
        if st:
            _lib.check(st)
        self.n_open -= 1

    def clone(self, stream_id: int, length: Optional[int] = None) -> int:
        """A new open stream beside ``stream_id`` (same parent and fork) that
        holds its first ``length`` tokens (default: all;
        ``padoc_session_clone``).  Blocks are shared until one of the streams
        appends to them."""
        if length is None:
            length = self._length(stream_id)
        i = C.c_int32(0)
        _lib.check(_lib.lib().padoc_session_clone(self.handle, int(stream_id), int(length), C.byref(i)))
        self.n_open += 1
        return int(i.value)

    def _length(self, stream_id: int) -> int:
        v = _lib.SessionView()
        _lib.check(_lib.lib().padoc_session_view_get(self.handle, C.byref(v)))
        at = np.nonzero(_carray(v.seg_id, v.n_seg, np.int32) == stream_id)[0]
        if len(at) == 0:
            raise ValueError(f"stream {stream_id} is not a kept stream of this session")
        return int(_carray(v.seg, v.n_seg, SEGMENT_DTYPE)["len"][at[0]])

    def truncate(self, stream_id: int, length: int) -> None:
        """Drop the tokens of an open stream behind its first ``length``
        (``padoc_session_truncate``)."""
        _lib.check(_lib.lib().padoc_session_truncate(self.handle, int(stream_id), int(length)))

    def compact(self, max_moves: int = 0) -> int:
        """Move kept blocks to the front of the pool, at most ``max_moves`` of
        them (0: all that it takes); the next launch copies them
        (``padoc_session_compact``).  Returns their number."""
        n = C.c_int32(0)
        _lib.check(_lib.lib().padoc_session_compact(self.handle, int(max_moves), C.byref(n)))
        return int(n.value)

    def resize(self, num_blocks: int, k_cache=None, v_cache=None) -> None:
        """Change the pool to ``num_blocks`` blocks
        (``padoc_session_resize``): with device caches, into ``k_cache`` /
        ``v_cache`` of that many blocks, which hold the present blocks at their
        ids (``k_cache[:num_blocks]`` of the old caches after a compaction, or
        larger ones the caller copied them to)."""
        if (k_cache is None) != (v_cache is None) or (k_cache is None) != (self.k_cache is None):
            raise ValueError("pass both caches, or neither for a host-only session")
        if k_cache is not None:
            got = _check_caches(k_cache, v_cache, self.k_cache.dtype, self.device)
            if got != (num_blocks, self.num_heads_kv, self.head_dim):
                raise ValueError(f"caches hold {got} blocks, heads and dimensions, expected "
                                 f"{(num_blocks, self.num_heads_kv, self.head_dim)}")
        _lib.check(_lib.lib().padoc_session_resize(self.handle, int(num_blocks),
                                                   None if k_cache is None else k_cache.data_ptr(),
                                                   None if v_cache is None else v_cache.data_ptr()))
        self.k_cache, self.v_cache, self.num_blocks = k_cache, v_cache, int(num_blocks)
        self._users = set()

    def copies(self):
        """The prepared step's block copies: one ``[n, 2]`` array of (source,
        destination) per phase (``padoc_session_copies``)."""
        n, ptr, pairs = C.c_int32(0), C.c_void_p(), C.c_void_p()
        _lib.check(_lib.lib().padoc_session_copies(self.handle, C.byref(n), C.byref(ptr), C.byref(pairs)))
        if n.value == 0:
            return []
        p = _carray(ptr.value, n.value + 1, np.int32)
        all_pairs = _carray(pairs.value, 2 * int(p[-1]), np.int32).reshape(-1, 2)
        return [all_pairs[a:b] for a, b in zip(p[:-1], p[1:])]

    def select(self, max_rows: int, priority=None):
        """``(n_new, n_query)`` for a step that takes at most ``max_rows``
        rows (``padoc_session_select``): the open streams with the largest
        ``priority`` (one entry per open stream, ascending id), or the oldest
        when ``priority`` is None."""
        n_new = np.zeros(self.n_open, np.int32)
        n_query = np.zeros(self.n_open, np.int32)
        pr = None
        if priority is not None:
            pr = np.ascontiguousarray(priority, dtype=np.int64)
            if pr.shape != (self.n_open,):
                raise ValueError(f"need one priority per open stream ({self.n_open}), got shape {pr.shape}")
        _lib.check(_lib.lib().padoc_session_select(self.handle, int(max_rows),
                                                   pr.ctypes.data if pr is not None and self.n_open else None,
                                                   n_new.ctypes.data, n_query.ctypes.data))
        return n_new, n_query

    def prepare(self, n_new=None, n_query=None):
        """Returns ``(n_kv_rows, n_q_rows, workspace_bytes)`` of the step."""
        arrs = []
        for a in (n_new, n_query):
            if a is None:
                arrs.append(None)
                continue
            a = np.ascontiguousarray(a, dtype=np.int32)
            if a.shape != (self.n_open,):
                raise ValueError(f"need one entry per open stream ({self.n_open}), got shape {a.shape}")
            arrs.append(a)
        if (arrs[0] is None) != (arrs[1] is None):
            raise ValueError("pass n_new and n_query together (or neither: one token and one query each)")
        nk, nq, ws = C.c_int32(0), C.c_int32(0), C.c_size_t(0)
        ptr = [a.ctypes.data if a is not None else None for a in arrs]
        _lib.check(_lib.lib().padoc_session_prepare(self.handle, ptr[0], ptr[1], C.byref(nk), C.byref(nq),
                                                    C.byref(ws)))
        self.n_kv_rows, self.n_q_rows, self.workspace_bytes = int(nk.value), int(nq.value), int(ws.value)
        return self.n_kv_rows, self.n_q_rows, self.workspace_bytes

    def workspace(self):
        """A cached device workspace of at least the prepared step's size."""
        import torch
        need = max(256, self.workspace_bytes)
        if self._ws is None or self._ws[2].numel() < need:
            cap = need + need // 4
            raw = torch.empty(cap + 256, dtype=torch.uint8, device=self.device)
            off = (-raw.data_ptr()) % 256
            self._ws = (self.device, raw, raw[off: off + cap])
            self._users = set()
        return self._ws[2]

    def _keep(self):
        """What the session holds belongs to the current stream, too, on which a
        step is about to use it: a workspace that the session outgrows, or caches
        that it is moved from, stay until the steps queued there are done."""
        import torch
        raw = torch._C._cuda_getCurrentRawStream(self.device.index)
        if raw in self._users:
            return
        s = torch.cuda.current_stream(self.device)
        for t in (self.k_cache, self.v_cache, self.block_table) + (() if self._ws is None else (self._ws[1],)):
            t.record_stream(s)
        self._users.add(raw)

    def launch(self, q, k_new, v_new, out=None, lse=None, workspace=None, stream=None):
        """Run the prepared step; q ``[n_q_rows, Hq, d]``, k_new / v_new
        ``[n_kv_rows, Hkv, d]``.  Returns ``(O, LSE)``."""
        import torch
        if self.device is None:
            raise RuntimeError("host-only session: use commit()")
        if stream is not None:
            return _on_stream(stream, self.device.index, self.launch, q, k_new, v_new, out, lse, workspace)
        dt = self.k_cache.dtype
        dev = self.device
        if self.n_kv_rows:
            for name, t in (("k_new", k_new), ("v_new", v_new)):
                _check_tensor(name, t, dt, dev)
                if tuple(t.shape) != (self.n_kv_rows, self.num_heads_kv, self.head_dim):
                    raise ValueError(f"{name} must be [{self.n_kv_rows}, {self.num_heads_kv}, {self.head_dim}]")
        if out is None:
            out = torch.empty(self.n_q_rows, self.num_heads_q, self.head_dim, dtype=dt, device=dev)
        if lse is None:
            lse = torch.empty(self.n_q_rows, self.num_heads_q, dtype=torch.float32, device=dev)
        if self.n_q_rows:
            _check_tensor("q", q, dt, dev)
            if tuple(q.shape) != (self.n_q_rows, self.num_heads_q, self.head_dim):
                raise ValueError(f"q must be [{self.n_q_rows}, {self.num_heads_q}, {self.head_dim}]")
            _check_tensor("out", out, dt, dev)
            _check_tensor("lse", lse, torch.float32, dev)
            if tuple(out.shape) != tuple(q.shape) or tuple(lse.shape) != tuple(q.shape[:2]):
                raise ValueError("out / lse shape does not match q")
        ws = self.workspace() if workspace is None else workspace
        self._keep()
        s = torch.cuda.current_stream(dev)

        def p(t, n):
            return _ptr(t) if n else None
        _lib.check(_lib.lib().padoc_session_launch(self.handle, p(q, self.n_q_rows), p(k_new, self.n_kv_rows),
                                                   p(v_new, self.n_kv_rows), p(out, self.n_q_rows),
                                                   p(lse, self.n_q_rows), _ptr(ws), ws.numel(),
                                                   C.c_void_p(s.cuda_stream)))
        return out, lse

    def launch_rotary(self, q, k_new, v_new, positions, rotary: Rotary, q_weight=None, k_weight=None, q_positions=None,
                      q_rot=None, out=None, lse=None, workspace=None, stream=None):
        """``launch`` for rows that are not rotated yet
        (``padoc_session_launch_rotary``): q, k_new and v_new are rows of the
        projections (they may be strided), ``positions`` int32 ``[n_axes,
        n_kv_rows]``; ``q_positions`` may be left out when every new token is a
        query.  ``q_rot`` receives the rotated queries (contiguous).  Returns
        ``(O, LSE)``."""
        import torch
        if self.device is None:
            raise RuntimeError("host-only session: use commit()")
        if stream is not None:
            return _on_stream(stream, self.device.index, self.launch_rotary, q, k_new, v_new, positions, rotary, q_weight,
                              k_weight, q_positions, q_rot, out, lse, workspace)
        n_q, n_kv = self.n_q_rows, self.n_kv_rows
        dt, dev = self.k_cache.dtype, self.device
        if _torch_dtype(rotary) != dt:
            raise TypeError(f"the rotary is for {rotary.dtype}, the session's caches are {dt}")
        if rotary.head_dim != self.head_dim:
            raise ValueError(f"the rotary is for heads of {rotary.head_dim}, the session's have {self.head_dim}")
        if n_kv:
            for name, t in (("k_new", k_new), ("v_new", v_new)):
                if not isinstance(t, torch.Tensor):
                    raise TypeError(f"{name} must be a torch tensor")
                if tuple(t.shape) != (n_kv, self.num_heads_kv, self.head_dim):
                    raise ValueError(f"{name} must be [{n_kv}, {self.num_heads_kv}, {self.head_dim}]")
        if n_q:
            if not isinstance(q, torch.Tensor):
                raise TypeError("q must be a torch tensor")
            if tuple(q.shape) != (n_q, self.num_heads_q, self.head_dim):
                raise ValueError(f"q must be [{n_q}, {self.num_heads_q}, {self.head_dim}]")
        if out is None:
            out = torch.empty(n_q, self.num_heads_q, self.head_dim, dtype=dt, device=dev)
        if lse is None:
            lse = torch.empty(n_q, self.num_heads_q, dtype=torch.float32, device=dev)
        if n_q:
            _check_tensor("out", out, dt, dev)
            _check_tensor("lse", lse, torch.float32, dev)
            if tuple(out.shape) != tuple(q.shape) or tuple(lse.shape) != tuple(q.shape[:2]):
                raise ValueError("out / lse shape does not match q")
            if q_rot is not None:
                _check_tensor("q_rot", q_rot, dt, dev)
        if n_q and n_kv and q_positions is None and n_q != n_kv:
            raise ValueError(f"{n_q} query rows of {n_kv} new ones need q_positions")
        if n_q or n_kv:
            args, _, device = _append_args(rotary, q if n_q else None, k_new if n_kv else None, v_new, positions,
                                             q_weight, k_weight, q_positions, q_rot)
            if device != dev.index:
                raise ValueError(f"rows are on cuda:{device}, expected {dev}")
        else:
            args = _lib.ROTARY_APPEND_ARGS.pack(*[0] * 26)
        # head counts are the session's also where a step has no rows of a kind
        args = args[:16] + struct.pack("=ii", self.num_heads_q, self.num_heads_kv) + args[24:]
        ws = self.workspace() if workspace is None else workspace
        self._keep()
        _launch(_lib.lib().padoc_session_launch_rotary, dev.index, self.handle, rotary.handle, args,
                out.data_ptr() if n_q else None, lse.data_ptr() if n_q else None, ws.data_ptr(), ws.numel())
        return out, lse

    def step(self, q, k_new, v_new, n_new=None, n_query=None, **kw):
        """``prepare`` then ``launch``."""
        self.prepare(n_new, n_query)
        return self.launch(q, k_new, v_new, **kw)

    def commit(self) -> None:
        _lib.check(_lib.lib().padoc_session_commit(self.handle))

    def view(self, schedule: bool = False, block_table: bool = True) -> dict:
        """The prepared step (or the tree as it stands) as numpy copies
        (``block_table=False`` skips copying the host block table)."""
        v = _lib.SessionView()
        _lib.check(_lib.lib().padoc_session_view_get(self.handle, C.byref(v)))
        arr = _carray
        n = v.n_rows
        prepared = bool(v.plan)
        out = {
            "seg": arr(v.seg, v.n_seg, SEGMENT_DTYPE), "seg_id": arr(v.seg_id, v.n_seg, np.int32),
            "row_id": arr(v.row_id, n, np.int32),
            "block_table": arr(v.block_table, self.block_table_capacity if block_table else 0, np.int32),
            "free_blocks": int(v.free_blocks), "prepared": prepared,
        }
        if prepared:
            new_off = arr(v.new_off, n + 1, np.int32)
            out.update({
                "new_off": new_off, "q_off": arr(v.q_off, n + 1, np.int32),
                "new_slot": arr(v.new_slot, 2 * int(new_off[-1]), np.int32).reshape(-1, 2),
                "patch": arr(v.patch, 2 * v.n_patch, np.int32).reshape(-1, 2),
                "workspace_bytes": int(v.workspace_bytes), "plan": int(v.plan),
            })
            if schedule:
                out["schedule"] = _export_schedule(C.c_void_p(v.plan))
        return out


def set_kernel_events(before=None, after=None):
    """Record torch CUDA events around all kernels of later calls on this
    thread (``padoc_set_kernel_events``); call with no arguments to stop."""
    b = C.c_void_p(before.cuda_event) if before is not None else None
    a = C.c_void_p(after.cuda_event) if after is not None else None
    _lib.check(_lib.lib().padoc_set_kernel_events(b, a))
