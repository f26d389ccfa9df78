"""ctypes binding of the operators around a paged cache (include/arkv_paged.h): argument marshalling and checks only.

Functions have the names of the C entry points; the descriptor structs have constructors that take tensors and keep them
alive.  What a call would index out of bounds with (shapes, types, devices) is checked here, with ValueError; what the C side
refuses raises binding.ArkvError.  Calls run on torch's current stream, allocate nothing and do not synchronise.
"""
from __future__ import annotations

import ctypes as C

from . import binding as _b
from .binding import ArkvError, EINVAL, EUNSUPPORTED, EHIP, OK  # noqa: F401

EXPORTED = ["arkv_paged_append", "arkv_paged_workspace", "arkv_paged_attention", "arkv_paged_weights", "arkv_paged_evict",
            "arkv_debug_paged_row"]


class _Pages(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("pos", C.c_void_p), ("weight", C.c_void_p)]


class _Batch(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_tokens", C.c_int32), ("max_q", C.c_int32), ("max_kv", C.c_int32),
                ("table_width", C.c_int32), ("cu_q", C.c_void_p), ("kv_len", C.c_void_p), ("table", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _Rotary(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("n_axes", C.c_int32), ("adjacent", C.c_int32), ("axis", C.c_uint8 * 64),
                ("freq", C.c_void_p)]


class _Scores(C.Structure):
    _fields_ = [("scale", C.c_float), ("cap", C.c_float), ("slopes", C.c_void_p), ("q_pos", C.c_void_p), ("prefix", C.c_void_p)]


_lib = None


def load():
    """libarkv.so with the signatures of these entry points."""
    global _lib
    if _lib is None:
        lib = _b.load()
        vp, i32, P = C.c_void_p, C.c_int32, C.POINTER
        pg, bt, sc, rw = P(_Pages), P(_Batch), P(_Scores), P(_Rows)
        sig = {
            "arkv_paged_append": [pg, bt, P(_Rotary), i32, rw, rw, rw, vp, vp, vp],
            "arkv_paged_workspace": [pg, bt, i32, P(C.c_size_t)],
            "arkv_paged_attention": [pg, bt, sc, i32, rw, vp, vp, vp, C.c_size_t, vp],
            "arkv_paged_weights": [pg, bt, sc, i32, rw, vp, C.c_float, vp, vp, C.c_size_t, vp],
            "arkv_paged_evict": [pg, bt, vp, i32, i32, i32, vp, i32, vp, vp, vp, C.c_size_t, vp],
            "arkv_debug_paged_row": [vp] + [i32] * 7 + [P(C.c_int64)],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = C.c_int, args
        _lib = lib
    return _lib


_TORCH = None


def _torch():
    global _TORCH
    import torch
    _b._lookup_torch()
    _TORCH = torch
    return torch


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _dense(t, shape, dtype, what, device=None):
    _need(t.is_cuda and t.is_contiguous(), f"{what}: a contiguous GPU tensor is needed")
    _need(t.dtype == dtype, f"{what}: expected {dtype}, got {t.dtype}")
    _need(tuple(t.shape) == tuple(shape), f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    _need(device is None or t.device == device, f"{what}: on {t.device}, the pages are on {device}")
    return t.data_ptr()


class arkv_pages:
    """One layer's pages: k, v [n_pages][H_kv][page_size][d] (bf16 or fp16), pos int32 and weight fp32 (or None)
    [n_pages][H_kv][page_size]."""

    def __init__(self, k, v, pos, weight=None):
        torch = _TORCH or _torch()
        _need(k.dim() == 4, "k: [n_pages][H_kv][page_size][d]")
        _need(k.dtype in (torch.bfloat16, torch.float16), f"k: bf16 or fp16, got {k.dtype}")
        self.k, self.v, self.pos, self.weight = k, v, pos, weight
        self.device, self.dtype = k.device, k.dtype
        self.n_pages, self.H, self.page_size, self.d = k.shape
        dev = k.device
        self.c = _Pages(0 if k.dtype == torch.bfloat16 else 1, self.n_pages, self.page_size, self.H, self.d,
                        _dense(k, k.shape, k.dtype, "k"), _dense(v, k.shape, k.dtype, "v", dev),
                        _dense(pos, k.shape[:3], torch.int32, "pos", dev),
                        None if weight is None else _dense(weight, k.shape[:3], torch.float32, "weight", dev))
        self.ref = C.byref(self.c)


class arkv_page_batch:
    """One step's sequences: cu_q int32 [B+1], kv_len int32 [B], table int32 [B][width] on the GPU; rows of the token-major
    tensors, and bounds of the sequences' new tokens and of their rows (None: as loose as the tensors allow)."""

    def __init__(self, cu_q, kv_len, table, n_tokens, max_q=None, max_kv=None, page_size=None):
        torch = _TORCH or _torch()
        _need(table.dim() == 2 and table.shape[0] >= 1, "table: [B][pages]")
        B, width = table.shape
        self.cu_q, self.kv_len, self.table = cu_q, kv_len, table
        self.device, self.B, self.n_tokens = table.device, B, n_tokens
        _need(max_kv is not None or page_size is not None, "max_kv or page_size is needed")
        self.c = _Batch(B, n_tokens, n_tokens if max_q is None else max_q, width * page_size if max_kv is None else max_kv, width,
                        _dense(cu_q, (B + 1,), torch.int32, "cu_q", table.device), _dense(kv_len, (B,), torch.int32, "kv_len", table.device),
                        _dense(table, (B, width), torch.int32, "table"))
        self.ref = C.byref(self.c)


class arkv_rotary:
    """freq fp64 [rot_dim / 2] on the GPU, radians per position; axis: which of n_axes positions turns pair i (None: the
    first); adjacent: pairs (2i, 2i+1) instead of (i, i + rot_dim / 2)."""

    def __init__(self, freq, axis=None, n_axes=1, adjacent=False):
        torch = _TORCH or _torch()
        half = 0 if freq is None else freq.numel()
        _need(half <= 64, "at most 64 pairs")
        axis = [0] * half if axis is None else [int(a) for a in axis]
        _need(len(axis) == half and all(0 <= a < 256 for a in axis), "axis: one entry per pair")
        self.freq, self.n_axes = freq, n_axes
        self.c = _Rotary(2 * half, n_axes, 1 if adjacent else 0, (C.c_uint8 * 64)(*axis),
                         None if freq is None else _dense(freq, (half,), torch.float64, "freq"))
        self.ref = C.byref(self.c)


def _rows(t, n, pages, what):
    """[n][heads][d] with any token and head stride; the channels are adjacent."""
    _need(t.is_cuda and t.dim() == 3 and t.shape[0] == n and t.shape[2] == pages.d, f"{what}: expected [{n}][heads][{pages.d}] on the GPU, got {tuple(t.shape)}")
    _need(t.dtype == pages.dtype and t.device == pages.device, f"{what}: expected {pages.dtype} on {pages.device}")
    _need(t.stride(2) == 1, f"{what}: channels must be adjacent")
    return C.byref(_Rows(t.data_ptr(), t.stride(0), t.stride(1)))


def _current(pages, batch):
    _need(batch.device == pages.device, "pages and batch are on different devices")
    _need(pages.device.index == _b._device(), f"the pages are on {pages.device}, which is not the current device")


def _workspace(ws, pages):
    if ws is None:
        return None, 0
    _need(ws.is_cuda and ws.is_contiguous() and ws.device == pages.device, "workspace: a contiguous tensor on the pages' device")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _call(name, *args):
    rc = getattr(_lib or load(), name)(*args)
    if rc != OK:
        raise ArkvError(rc, name)


# ---- entry points, same names as the C ABI -----------------------------------------------------

def arkv_paged_workspace(pages, batch, n_q_heads):
    """A workspace tensor for the calls below (uint8; allocate once for the largest batch)."""
    torch = _TORCH or _torch()
    n = C.c_size_t()
    _call("arkv_paged_workspace", pages.ref, batch.ref, n_q_heads, C.byref(n))
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device=pages.device)


def arkv_paged_append(pages, batch, rotary, q, k, v, positions, q_out):
    """q [n][H_q][d], k, v [n][H_kv][d] (strided), positions int32 [n_axes][n]; q and q_out may both be None."""
    torch = _TORCH or _torch()
    _current(pages, batch)
    n, H = batch.n_tokens, pages.H
    _need(k.shape[1] == H and v.shape[1] == H, f"k, v: expected {H} heads")
    _need(rotary.freq is None or rotary.freq.device == pages.device, "freq: on another device than the pages")
    hq = 0
    if q is not None or q_out is not None:
        _need(q is not None and q_out is not None, "q and q_out go together")
        hq = q.shape[1]
    _call("arkv_paged_append", pages.ref, batch.ref, rotary.ref, hq, None if q is None else _rows(q, n, pages, "q"),
          _rows(k, n, pages, "k"), _rows(v, n, pages, "v"),
          _dense(positions, (rotary.n_axes, n), torch.int32, "positions", pages.device),
          None if q is None else _dense(q_out, (n, hq, pages.d), pages.dtype, "q_out", pages.device), _b._stream())


def _scores(pages, batch, hq, scale, cap, slopes, q_pos, prefix):
    torch = _TORCH
    s = _Scores(scale, cap, None, None, None)
    if slopes is not None:
        _need(q_pos is not None, "slopes need q_pos")
        s.slopes = _dense(slopes, (hq,), torch.float32, "slopes", pages.device)
        s.q_pos = _dense(q_pos, (batch.n_tokens,), torch.int32, "q_pos", pages.device)
    if prefix is not None:
        s.prefix = _dense(prefix, (batch.B,), torch.int32, "prefix", pages.device)
    return C.byref(s)


def arkv_paged_attention(pages, batch, q, scale, out, lse=None, cap=0.0, slopes=None, q_pos=None, prefix=None, workspace=None):
    """q [n][H_q][d] (strided), out [n][H_q][d], lse fp32 [n][H_q] or None; the other arguments as arkv_scores."""
    torch = _TORCH or _torch()
    _current(pages, batch)
    n, hq = batch.n_tokens, q.shape[1]
    ws, size = _workspace(workspace, pages)
    _call("arkv_paged_attention", pages.ref, batch.ref, _scores(pages, batch, hq, scale, cap, slopes, q_pos, prefix), hq,
          _rows(q, n, pages, "q"), _dense(out, (n, hq, pages.d), pages.dtype, "out", pages.device),
          None if lse is None else _dense(lse, (n, hq), torch.float32, "lse", pages.device), ws, size, _b._stream())


def arkv_paged_weights(pages, batch, q, scale, lse, decay=1.0, carried=None, cap=0.0, slopes=None, q_pos=None, prefix=None,
                       workspace=None):
    """Adds the tokens' probabilities to pages.weight (decay * carried + sum); carried None: pages.weight itself."""
    torch = _TORCH or _torch()
    _current(pages, batch)
    n, hq = batch.n_tokens, q.shape[1]
    ws, size = _workspace(workspace, pages)
    _call("arkv_paged_weights", pages.ref, batch.ref, _scores(pages, batch, hq, scale, cap, slopes, q_pos, prefix), hq,
          _rows(q, n, pages, "q"), _dense(lse, (n, hq), torch.float32, "lse", pages.device), decay,
          None if carried is None else _dense(carried, (pages.n_pages, pages.H, pages.page_size), torch.float32, "carried", pages.device),
          ws, size, _b._stream())


def arkv_paged_evict(pages, batch, keep, dst_table, kept, new_len, sink=4, recent=32, workspace=None):
    """keep int32 [B], dst_table int32 [B][pages], kept int32 [B][H_kv][max_keep] (out), new_len int32 [B] (out)."""
    torch = _TORCH or _torch()
    _current(pages, batch)
    B = batch.B
    _need(dst_table.dim() == 2 and kept.dim() == 3, "dst_table: [B][pages]; kept: [B][H_kv][max_keep]")
    width, max_keep = dst_table.shape[1], kept.shape[2]
    ws, size = _workspace(workspace, pages)
    _call("arkv_paged_evict", pages.ref, batch.ref, _dense(keep, (B,), torch.int32, "keep", pages.device), max_keep, sink, recent,
          _dense(dst_table, (B, width), torch.int32, "dst_table", pages.device), width,
          _dense(kept, (B, pages.H, max_keep), torch.int32, "kept", pages.device),
          _dense(new_len, (B,), torch.int32, "new_len", pages.device), ws, size, _b._stream())


def arkv_debug_paged_row(table_row, n_pages, page_size, n_kv_heads, kv_head, length, slot):
    """Row of [n_pages][H_kv][page_size] in which the kernels look for a slot, -1: none.  table_row: NumPy int32."""
    import numpy as np
    t = np.ascontiguousarray(table_row, dtype=np.int32)
    row = C.c_int64()
    _call("arkv_debug_paged_row", t.ctypes.data_as(C.c_void_p), len(t), n_pages, page_size, n_kv_heads, kv_head, length, slot,
          C.byref(row))
    return row.value
