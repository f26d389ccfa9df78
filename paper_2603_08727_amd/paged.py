"""ctypes binding of the operators around a paged cache (include/arkv_paged.h): argument marshalling and checks only.

Functions have the names of the C entry points; the descriptor structs have constructors that take tensors and keep them
alive.  What a call would index out of bounds with (shapes, types, devices) is checked here, with ValueError; what the C side
refuses raises binding.ArkvError.  Calls run on torch's current stream, allocate nothing and do not synchronise.
"""
from __future__ import annotations

import ctypes as C
import threading

from . import binding as _b
from .binding import ArkvError, EINVAL, EUNSUPPORTED, EHIP, OK  # noqa: F401

TICKET_BYTES = 1 << 16                             # of a workspace's front, zero between calls

EXPORTED = ["arkv_paged_append", "arkv_paged_workspace", "arkv_paged_attention", "arkv_paged_weights", "arkv_paged_evict",
            "arkv_paged_attention_sight", "arkv_packed_append", "arkv_packed_read", "arkv_packed_workspace", "arkv_packed_attention",
            "arkv_debug_paged_row", "arkv_debug_attention_cut"]


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


class _Sight(C.Structure):
    _fields_ = [("window", C.c_int32), ("sink", C.c_int32), ("tree_words", C.c_int32), ("tree", C.c_void_p)]


class _Packed(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("bits", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("pos", C.c_void_p)]


_lib = None


def load():
    """libarkv.so with the signatures of these entry points."""
    global _lib
    if _lib is None:
        lib = _b.load()
        vp, i32 = C.c_void_p, C.c_int32
        pg = bt = sc = rw = rt = vp            # (structs go as plain addresses: ctypes checks a pointer type in 0.1 us each)
        sig = {
            "arkv_paged_append": [pg, bt, rt, i32, rw, rw, rw, vp, vp, vp],
            "arkv_paged_workspace": [pg, bt, i32, vp],
            "arkv_paged_attention": [pg, bt, sc, i32, rw, vp, vp, vp, C.c_size_t, vp],
            "arkv_paged_weights": [pg, bt, sc, i32, rw, vp, C.c_float, vp, vp, C.c_size_t, vp],
            "arkv_paged_evict": [pg, bt, vp, i32, i32, i32, vp, i32, vp, vp, vp, C.c_size_t, vp],
            "arkv_paged_attention_sight": [pg, bt, sc, vp, i32, rw, vp, vp, vp, C.c_size_t, vp],
            "arkv_packed_append": [pg, bt, rt, i32, rw, rw, rw, vp, vp, vp],
            "arkv_packed_read": [pg, bt, vp, vp, vp],
            "arkv_packed_workspace": [pg, bt, i32, vp],
            "arkv_packed_attention": [pg, bt, sc, vp, i32, rw, vp, vp, vp, C.c_size_t, vp],
            "arkv_debug_paged_row": [vp] + [i32] * 7 + [vp],
            "arkv_debug_attention_cut": [pg, bt, sc, vp, i32, vp],
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


def _int32(**numbers):
    """Python's numbers have no end; ctypes would pass on their lowest 32 bits."""
    for what, x in numbers.items():
        if not -2 ** 31 <= x < 2 ** 31:
            raise ValueError(f"{what}: {x} does not fit 32 bits")


def _dense(t, shape, dtype, what, index=None):
    """Address of a contiguous GPU tensor (on GPU `index`) of that shape and type."""
    at = t.get_device()
    if t.shape != shape or t.dtype is not dtype or at != (at if index is None else index) or at < 0 or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on the pages' GPU, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class arkv_pages:
    """One layer's pages: k, v [n_pages][H_kv][page_size][d] (bf16 or fp16), pos int32 and weight fp32 (or None)
    [n_pages][H_kv][page_size]."""

    def __init__(self, k, v, pos, weight=None):
        torch = _TORCH or _torch()
        _need(k.dim() == 4, "k: [n_pages][H_kv][page_size][d]")
        _need(k.dtype in (torch.bfloat16, torch.float16), f"k: bf16 or fp16, got {k.dtype}")
        self.k, self.v, self.pos, self.weight = k, v, pos, weight
        self.device, self.dtype, self.index = k.device, k.dtype, k.get_device()
        self.n_pages, self.H, self.page_size, self.d = k.shape
        self.rows = k.shape[:3]
        dev = self.index
        self.c = _Pages(0 if k.dtype == torch.bfloat16 else 1, self.n_pages, self.page_size, self.H, self.d,
                        _dense(k, k.shape, k.dtype, "k"), _dense(v, k.shape, k.dtype, "v", dev),
                        _dense(pos, k.shape[:3], torch.int32, "pos", dev),
                        None if weight is None else _dense(weight, k.shape[:3], torch.float32, "weight", dev))
        self.ref = C.addressof(self.c)


class arkv_packed_pages:
    """One layer's packed pages: k, v uint8 [n_pages][H_kv][page_size][d * bits / 8], k_scale, v_scale uint8
    [n_pages][H_kv][page_size][d / 32] (their width says d, and with it bits), pos int32 [n_pages][H_kv][page_size]; dtype: bf16 or
    fp16, of the rows that go in and come out."""

    def __init__(self, k, v, k_scale, v_scale, pos, dtype):
        torch = _TORCH or _torch()
        _need(k.dim() == 4 and k_scale.dim() == 4, "k: [n_pages][H_kv][page_size][bytes], k_scale: [n_pages][H_kv][page_size][d / 32]")
        _need(dtype in (torch.bfloat16, torch.float16), f"dtype: bf16 or fp16, got {dtype}")
        self.k, self.v, self.k_scale, self.v_scale, self.pos = k, v, k_scale, v_scale, pos
        self.device, self.dtype, self.index = k.device, dtype, k.get_device()
        self.n_pages, self.H, self.page_size, width = k.shape
        self.rows, self.d = k.shape[:3], 32 * k_scale.size(3)
        _need(width in (self.d, self.d // 2), f"k: {width} bytes for {self.d} channels: 8 or 4 bits each")
        self.bits = 8 if width == self.d else 4
        dev, u8, scales = self.index, torch.uint8, (*self.rows, self.d // 32)
        self.c = _Packed(0 if dtype == torch.bfloat16 else 1, self.bits, self.n_pages, self.page_size, self.H, self.d,
                         _dense(k, k.shape, u8, "k"), _dense(v, k.shape, u8, "v", dev), _dense(k_scale, scales, u8, "k_scale", dev),
                         _dense(v_scale, scales, u8, "v_scale", dev), _dense(pos, self.rows, torch.int32, "pos", dev))
        self.ref = C.addressof(self.c)


class arkv_sight:
    """Which slots a new token sees: window rows back (0: all) and the first `sink`; of the new tokens those whose bits in tree say so
    (int64 or uint64 [n_tokens][words] on the GPU; None: those up to itself)."""

    def __init__(self, window=0, sink=0, tree=None):
        torch = _TORCH or _torch()
        _int32(window=window, sink=sink)
        words = 0
        if tree is not None:
            _need(tree.dim() == 2 and tree.dtype in (torch.int64, torch.uint64), f"tree: int64 or uint64 [n_tokens][words], got {tree.dtype} {tuple(tree.shape)}")
            words = tree.size(1)
            _need(words >= 1, "tree: at least one word a token")       # (a tensor of nothing has no address: it would be no tree)
        self.tree, self.n_tokens, self.index = tree, None if tree is None else tree.size(0), None if tree is None else tree.get_device()
        self.c = _Sight(window, sink, words, None if tree is None else _dense(tree, tree.shape, tree.dtype, "tree"))
        self.ref = C.addressof(self.c)


class arkv_page_batch:
    """One step's sequences: cu_q int32 [B+1], kv_len int32 [B], table int32 [B][width] on the GPU; rows of the token-major
    tensors, and bounds of the sequences' new tokens and of their rows (None: as loose as the tensors allow)."""

    def __init__(self, cu_q, kv_len, table, n_tokens, max_q=None, max_kv=None, page_size=None):
        torch = _TORCH or _torch()
        _need(table.dim() == 2 and table.shape[0] >= 1, "table: [B][pages]")
        B, width = table.shape
        self.cu_q, self.kv_len, self.table = cu_q, kv_len, table
        self.device, self.index, self.B, self.n_tokens = table.device, table.get_device(), B, n_tokens
        _need(max_kv is not None or page_size is not None, "max_kv or page_size is needed")
        max_q, max_kv = n_tokens if max_q is None else max_q, width * page_size if max_kv is None else max_kv
        _int32(n_tokens=n_tokens, max_q=max_q, max_kv=max_kv)
        self.c = _Batch(B, n_tokens, max_q, max_kv, width,
                        _dense(cu_q, (B + 1,), torch.int32, "cu_q", self.index), _dense(kv_len, (B,), torch.int32, "kv_len", self.index),
                        _dense(table, (B, width), torch.int32, "table"))
        self.ref = C.addressof(self.c)


class arkv_rotary:
    """freq fp64 [rot_dim / 2] on the GPU, radians per position; axis: which of n_axes positions turns pair i (None: the
    first); adjacent: pairs (2i, 2i+1) instead of (i, i + rot_dim / 2)."""

    def __init__(self, freq, axis=None, n_axes=1, adjacent=False):
        torch = _TORCH or _torch()
        half = 0 if freq is None else freq.numel()
        _need(half <= 64, "at most 64 pairs")
        axis = [0] * half if axis is None else [int(a) for a in axis]
        _need(len(axis) == half and all(0 <= a < 256 for a in axis), "axis: one entry per pair")
        _int32(n_axes=n_axes)
        self.freq, self.n_axes, self.index = freq, n_axes, None if freq is None else freq.get_device()
        self.c = _Rotary(2 * half, n_axes, 1 if adjacent else 0, (C.c_uint8 * 64)(*axis),
                         None if freq is None else _dense(freq, (half,), torch.float64, "freq"))
        self.ref = C.addressof(self.c)


# A call's own structs.  Making one costs a microsecond, so every thread keeps its set and fills it anew in each call (the C
# side reads them before it returns).
class _Set:
    def __init__(self):
        self.q, self.k, self.v, self.s, self.plain = _Rows(), _Rows(), _Rows(), _Scores(), _Scores()   # (plain: no arrays)
        self.rq, self.rk, self.rv, self.rs, self.rplain = (C.addressof(x) for x in (self.q, self.k, self.v, self.s, self.plain))


class _Own(threading.local):
    def __init__(self):
        self.set = _Set()


_own = _Own()


def _rows(to, t, n, pages, what):
    """[n][heads][d] with any token and head stride; the channels are adjacent.  Returns the number of heads."""
    shape = t.shape
    if len(shape) == 3:
        tokens, heads, channels = shape
        if tokens == n and channels == pages.d and t.dtype is pages.dtype and t.get_device() == pages.index:
            to.token_stride, to.head_stride, channel = t.stride()
            if channel != 1:
                raise ValueError(f"{what}: channels must be adjacent")
            if tokens == 1:                            # (a stride that nothing is multiplied by can be any number in torch)
                to.token_stride = 0
            if heads == 1:
                to.head_stride = 0
            to.p = t.data_ptr()
            return heads
    raise ValueError(f"{what}: expected {pages.dtype} [{n}][heads][{pages.d}] on {pages.device}, got {t.dtype} {tuple(shape)} on {t.device}")


def _kind(pages, kind):
    """A struct of the other kind of pages would be read with its fields moved."""
    if not isinstance(pages, kind):
        raise ValueError(f"pages: expected {kind.__name__}, got {type(pages).__name__}")


def _current(pages, batch, kind):
    """Handle of torch's current stream on the device where everything has to be."""
    if not isinstance(pages, kind):
        _kind(pages, kind)
    at = pages.index
    if batch.index != at or at != _b._device():
        raise ValueError(f"pages on {pages.device}, batch on {batch.device}: both must be on the current device")
    return _b._raw_stream(at)


def _workspace(ws, pages):
    if ws is None:
        return None, 0
    if ws.get_device() != pages.index or not ws.is_contiguous():
        raise ValueError("workspace: a contiguous tensor on the pages' device")
    return ws.data_ptr(), ws.nbytes


def _check(rc, name):
    if rc != OK:
        raise ArkvError(rc, name)


# ---- entry points, same names as the C ABI -----------------------------------------------------

def arkv_paged_workspace_bytes(pages, batch, n_q_heads):
    """Bytes of workspace that the calls below need for this batch, or any with no more sequences, tokens, new tokens or rows."""
    _kind(pages, arkv_pages)
    n = C.c_size_t()
    _check((_lib or load()).arkv_paged_workspace(pages.ref, batch.ref, n_q_heads, C.addressof(n)), "arkv_paged_workspace")
    return n.value


def arkv_paged_workspace(pages, batch, n_q_heads):
    """A workspace tensor for the calls below, its front zeroed as its first use wants it; one for the largest of each of a batch's
    bounds (sequences, n_tokens, max_q, max_kv) serves all."""
    torch = _TORCH or _torch()
    ws = torch.empty(arkv_paged_workspace_bytes(pages, batch, n_q_heads), dtype=torch.uint8, device=pages.device)
    ws[:TICKET_BYTES].zero_()
    return ws


def _append(name, torch, stream, pages, batch, rotary, q, k, v, positions, q_out):
    n, H, o = batch.n_tokens, pages.H, _own.set
    if rotary.index != pages.index and rotary.index is not None:
        raise ValueError("freq: on another device than the pages")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if _rows(o.k, k, n, pages, "k") != H or _rows(o.v, v, n, pages, "v") != H:
        raise ValueError(f"k, v: expected {H} heads")
    hq, rq, to = 0, None, None
    if q is not None:
        hq, rq = _rows(o.q, q, n, pages, "q"), o.rq
        to = _dense(q_out, (n, hq, pages.d), pages.dtype, "q_out", pages.index)
    rc = getattr(_lib or load(), name)(pages.ref, batch.ref, rotary.ref, hq, rq, o.rk, o.rv,
                                       _dense(positions, (rotary.n_axes, n), torch.int32, "positions", pages.index), to, stream)
    _check(rc, name)


def arkv_paged_append(pages, batch, rotary, q, k, v, positions, q_out):
    """q [n][H_q][d], k, v [n][H_kv][d] (strided), positions int32 [n_axes][n]; q and q_out may both be None."""
    torch = _TORCH or _torch()
    _append("arkv_paged_append", torch, _current(pages, batch, arkv_pages), pages, batch, rotary, q, k, v, positions, q_out)


def _scores(o, pages, batch, hq, scale, cap, slopes, q_pos, prefix):
    if slopes is None and prefix is None:
        o.plain.scale, o.plain.cap = scale, cap
        return o.rplain
    torch, s = _TORCH, o.s
    s.scale, s.cap, s.slopes, s.q_pos, s.prefix = scale, cap, None, None, None
    if slopes is not None:
        if q_pos is None:
            raise ValueError("slopes need q_pos")
        s.slopes = _dense(slopes, (hq,), torch.float32, "slopes", pages.index)
        s.q_pos = _dense(q_pos, (batch.n_tokens,), torch.int32, "q_pos", pages.index)
    if prefix is not None:
        s.prefix = _dense(prefix, (batch.B,), torch.int32, "prefix", pages.index)
    return o.rs


def arkv_paged_attention(pages, batch, q, scale, out, lse=None, cap=0.0, slopes=None, q_pos=None, prefix=None, workspace=None):
    """q [n][H_q][d] (strided), out [n][H_q][d], lse fp32 [n][H_q] or None; the other arguments as arkv_scores."""
    torch = _TORCH or _torch()
    stream = _current(pages, batch, arkv_pages)
    n, o, at = batch.n_tokens, _own.set, pages.index
    hq = _rows(o.q, q, n, pages, "q")
    ws, size = _workspace(workspace, pages)
    rc = (_lib or load()).arkv_paged_attention(
        pages.ref, batch.ref, _scores(o, pages, batch, hq, scale, cap, slopes, q_pos, prefix), hq, o.rq,
        _dense(out, (n, hq, pages.d), pages.dtype, "out", at), None if lse is None else _dense(lse, (n, hq), torch.float32, "lse", at),
        ws, size, stream)
    _check(rc, "arkv_paged_attention")


def _sight(sight, pages, batch):
    if sight is None:
        return None
    if sight.tree is not None and (sight.n_tokens != batch.n_tokens or sight.index != pages.index):
        raise ValueError(f"tree: expected {batch.n_tokens} tokens on {pages.device}, got {sight.n_tokens} on {sight.tree.device}")
    return sight.ref


def arkv_paged_attention_sight(pages, batch, sight, q, scale, out, lse=None, cap=0.0, slopes=None, q_pos=None, prefix=None, workspace=None):
    """arkv_paged_attention with an arkv_sight."""
    torch = _TORCH or _torch()
    stream = _current(pages, batch, arkv_pages)
    n, o, at = batch.n_tokens, _own.set, pages.index
    hq = _rows(o.q, q, n, pages, "q")
    ws, size = _workspace(workspace, pages)
    rc = (_lib or load()).arkv_paged_attention_sight(
        pages.ref, batch.ref, _scores(o, pages, batch, hq, scale, cap, slopes, q_pos, prefix), _sight(sight, pages, batch), hq, o.rq,
        _dense(out, (n, hq, pages.d), pages.dtype, "out", at), None if lse is None else _dense(lse, (n, hq), torch.float32, "lse", at),
        ws, size, stream)
    _check(rc, "arkv_paged_attention_sight")


def arkv_packed_append(pages, batch, rotary, q, k, v, positions, q_out):
    """arkv_paged_append into packed pages."""
    torch = _TORCH or _torch()
    _append("arkv_packed_append", torch, _current(pages, batch, arkv_packed_pages), pages, batch, rotary, q, k, v, positions, q_out)


def arkv_packed_read(pages, batch, k, v):
    """k, v [n][H_kv][d] (out; either may be None): the values of the batch's new tokens' rows."""
    _TORCH or _torch()
    stream = _current(pages, batch, arkv_packed_pages)
    shape = (batch.n_tokens, pages.H, pages.d)
    k, v = (None if x is None else _dense(x, shape, pages.dtype, what, pages.index) for x, what in ((k, "k"), (v, "v")))
    _check((_lib or load()).arkv_packed_read(pages.ref, batch.ref, k, v, stream), "arkv_packed_read")


def arkv_packed_workspace_bytes(pages, batch, n_q_heads):
    """Bytes of workspace that arkv_packed_attention needs for this batch, or any with no more sequences, tokens, new tokens or rows."""
    _kind(pages, arkv_packed_pages)
    n = C.c_size_t()
    _check((_lib or load()).arkv_packed_workspace(pages.ref, batch.ref, n_q_heads, C.addressof(n)), "arkv_packed_workspace")
    return n.value


def arkv_packed_workspace(pages, batch, n_q_heads):
    """A workspace tensor for arkv_packed_attention, as arkv_paged_workspace makes one."""
    torch = _TORCH or _torch()
    ws = torch.empty(arkv_packed_workspace_bytes(pages, batch, n_q_heads), dtype=torch.uint8, device=pages.device)
    ws[:TICKET_BYTES].zero_()
    return ws


def arkv_packed_attention(pages, batch, q, scale, out, lse=None, cap=0.0, slopes=None, q_pos=None, prefix=None, sight=None, workspace=None):
    """arkv_paged_attention over the values of packed rows; sight: an arkv_sight, or None."""
    torch = _TORCH or _torch()
    stream = _current(pages, batch, arkv_packed_pages)
    n, o, at = batch.n_tokens, _own.set, pages.index
    hq = _rows(o.q, q, n, pages, "q")
    ws, size = _workspace(workspace, pages)
    rc = (_lib or load()).arkv_packed_attention(
        pages.ref, batch.ref, _scores(o, pages, batch, hq, scale, cap, slopes, q_pos, prefix), _sight(sight, pages, batch), hq, o.rq,
        _dense(out, (n, hq, pages.d), pages.dtype, "out", at), None if lse is None else _dense(lse, (n, hq), torch.float32, "lse", at),
        ws, size, stream)
    _check(rc, "arkv_packed_attention")


def arkv_paged_weights(pages, batch, q, scale, lse, decay=1.0, carried=None, cap=0.0, slopes=None, q_pos=None, prefix=None,
                       workspace=None):
    """Adds the tokens' probabilities to pages.weight (decay * carried + sum); carried None: pages.weight itself."""
    torch = _TORCH or _torch()
    stream = _current(pages, batch, arkv_pages)
    n, o, at = batch.n_tokens, _own.set, pages.index
    hq = _rows(o.q, q, n, pages, "q")
    ws, size = _workspace(workspace, pages)
    rc = (_lib or load()).arkv_paged_weights(
        pages.ref, batch.ref, _scores(o, pages, batch, hq, scale, cap, slopes, q_pos, prefix), hq, o.rq,
        _dense(lse, (n, hq), torch.float32, "lse", at), decay, None if carried is None else _dense(carried, pages.rows, torch.float32, "carried", at),
        ws, size, stream)
    _check(rc, "arkv_paged_weights")


def arkv_paged_evict(pages, batch, keep, dst_table, kept, new_len, sink=4, recent=32, workspace=None):
    """keep int32 [B], dst_table int32 [B][pages], kept int32 [B][H_kv][max_keep] (out), new_len int32 [B] (out)."""
    torch = _TORCH or _torch()
    stream = _current(pages, batch, arkv_pages)
    B, at, i32 = batch.B, pages.index, torch.int32
    _need(dst_table.dim() == 2 and kept.dim() == 3, "dst_table: [B][pages]; kept: [B][H_kv][max_keep]")
    _int32(sink=sink, recent=recent)
    width, max_keep = dst_table.size(1), kept.size(2)
    ws, size = _workspace(workspace, pages)
    rc = (_lib or load()).arkv_paged_evict(
        pages.ref, batch.ref, _dense(keep, (B,), i32, "keep", at), max_keep, sink, recent, _dense(dst_table, (B, width), i32, "dst_table", at), width,
        _dense(kept, (B, pages.H, max_keep), i32, "kept", at), _dense(new_len, (B,), i32, "new_len", at), ws, size, stream)
    _check(rc, "arkv_paged_evict")


def arkv_debug_paged_row(table_row, n_pages, page_size, n_kv_heads, kv_head, length, slot):
    """Row of [n_pages][H_kv][page_size] in which the kernels look for a slot, -1: none.  table_row: NumPy int32."""
    import numpy as np
    _int32(n_pages=n_pages, page_size=page_size, n_kv_heads=n_kv_heads, kv_head=kv_head, length=length, slot=slot)
    t = np.ascontiguousarray(table_row, dtype=np.int32)
    row = C.c_int64()
    _check((_lib or load()).arkv_debug_paged_row(t.ctypes.data, len(t), n_pages, page_size, n_kv_heads, kv_head, length, slot, C.addressof(row)),
           "arkv_debug_paged_row")
    return row.value


def arkv_debug_attention_cut(cu_q, kv_len, n_tokens, max_q, max_kv, n_q_heads, n_kv_heads, head_dim, bits, window=0, sink=0, tree_words=0, cap=0.0,
                             prefix=None):
    """How an attention call over pages of 16-, 8- or 4-bit rows divides a batch: the nine numbers of the header's text.  cu_q, kv_len, prefix: NumPy
    int32; tree_words: 0 without a tree."""
    import numpy as np
    _int32(n_tokens=n_tokens, max_q=max_q, max_kv=max_kv, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, window=window, sink=sink)
    cu_q, kv_len, prefix = (None if x is None else np.ascontiguousarray(x, dtype=np.int32) for x in (cu_q, kv_len, prefix))
    B, cut, none = len(kv_len), (C.c_int32 * 9)(), 16      # (an address that is not followed)
    _need(len(cu_q) == B + 1 and (prefix is None or len(prefix) == B), "cu_q: [B + 1], kv_len, prefix: [B]")
    pages = _Packed(0, bits, 1, 16, n_kv_heads, head_dim, none, none, none, none, none)
    batch = _Batch(B, n_tokens, max_q, max_kv, max(1, -(-max_kv // 16)), cu_q.ctypes.data, kv_len.ctypes.data, none)
    scores = _Scores(1.0, cap, None, None, None if prefix is None else prefix.ctypes.data)
    sight = _Sight(window, sink, tree_words, none if tree_words else None)
    _check((_lib or load()).arkv_debug_attention_cut(*(C.addressof(x) for x in (pages, batch, scores, sight)), n_q_heads, cut), "arkv_debug_attention_cut")
    return list(cut)
