"""CPU checks of the paged operators' entry points: exports, refusals before anything is launched, slots of pages."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from paper_2603_08727_amd import binding as A
from paper_2603_08727_amd import paged as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_header_binding_and_library_agree():
    hdr = open(os.path.join(ROOT, "include", "arkv_paged.h")).read()
    hdr = re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)
    declared = set(re.findall(r"\b(arkv_[a-z0-9_]+)\s*\(", hdr))
    assert declared == set(P.EXPORTED)
    lib = P.load()
    for name in declared:
        assert hasattr(lib, name), name


@pytest.mark.parametrize("page,hkv", [(16, 1), (16, 3), (64, 8), (1024, 2)])
def test_slots_of_pages(page, hkv):
    rng = np.random.default_rng(page + hkv)
    n_pages, width = 50, 7
    table = rng.permutation(n_pages)[:width].astype(np.int32)
    table[2], table[4] = -1, n_pages
    length = width * page - 5
    for slot in [-2**31, -1, 0, 1, page - 1, page, 2 * page, 3 * page - 1, 4 * page, length - 1, length, width * page, 2**31 - 1]:
        for h in (0, hkv - 1):
            got = P.arkv_debug_paged_row(table, n_pages, page, hkv, h, length, slot)
            if not 0 <= slot < length or slot // page in (2, 4):
                assert got == -1
            else:
                assert got == (int(table[slot // page]) * hkv + h) * page + slot % page


def test_slot_hook_refusals():
    t = np.zeros(4, np.int32)
    for bad in [dict(n_pages=0), dict(page=8), dict(page=24), dict(page=2048), dict(hkv=0), dict(h=1), dict(h=-1), dict(length=-1),
                dict(length=65)]:
        kw = dict(n_pages=4, page=16, hkv=1, h=0, length=64)
        kw.update(bad)
        with pytest.raises(A.ArkvError) as e:
            P.arkv_debug_paged_row(t, kw["n_pages"], kw["page"], kw["hkv"], kw["h"], kw["length"], 0)
        assert e.value.code == A.EINVAL
    assert P.load().arkv_debug_paged_row(None, 4, 4, 16, 1, 0, 4, 0, None) == A.EINVAL


# Addresses that are never followed: every call below is refused on the host.
ADDR = 0x1000


def _args():
    pages = P._Pages(0, 100, 16, 2, 64, ADDR, ADDR, ADDR, ADDR)
    batch = P._Batch(2, 10, 5, 64, 4, ADDR, ADDR, ADDR)
    rows = P._Rows(ADDR, 512, 64)
    rot = P._Rotary(64, 1, 0, (C.c_uint8 * 64)(), ADDR)
    sc = P._Scores(0.125, 0.0, None, None, None)
    return pages, batch, rows, rot, sc


def _call(name, pages, batch, rows, rot, sc, hq=8, ws=ADDR, size=1 << 40, **kw):
    lib = P.load()
    r = C.byref
    if name == "append":
        return lib.arkv_paged_append(r(pages), r(batch), r(rot), hq, r(rows), r(rows), r(rows), kw.get("positions", ADDR), kw.get("out", ADDR), None)
    if name == "workspace":
        return lib.arkv_paged_workspace(r(pages), r(batch), hq, r(C.c_size_t()))
    if name == "attention":
        return lib.arkv_paged_attention(r(pages), r(batch), r(sc), hq, r(rows), kw.get("out", ADDR), None, ws, size, None)
    if name == "weights":
        return lib.arkv_paged_weights(r(pages), r(batch), r(sc), hq, r(rows), kw.get("lse", ADDR), kw.get("decay", 1.0), None, ws, size, None)
    return lib.arkv_paged_evict(r(pages), r(batch), kw.get("keep", ADDR), kw.get("max_keep", 32), kw.get("sink", 4), kw.get("recent", 8),
                                kw.get("dst", ADDR), kw.get("dst_width", 2), kw.get("kept", ADDR), kw.get("new_len", ADDR), ws, size, None)


ALL = ["append", "workspace", "attention", "weights", "evict"]


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("where,field,value,code", [
    ("pages", "k", None, A.EINVAL), ("pages", "v", None, A.EINVAL), ("pages", "pos", None, A.EINVAL), ("pages", "n_pages", 0, A.EINVAL),
    ("pages", "n_pages", -3, A.EINVAL), ("pages", "page_size", 0, A.EINVAL), ("pages", "page_size", 24, A.EINVAL),
    ("pages", "page_size", 8, A.EUNSUPPORTED), ("pages", "page_size", 2048, A.EUNSUPPORTED), ("pages", "n_kv_heads", 0, A.EINVAL),
    ("pages", "head_dim", 96, A.EUNSUPPORTED), ("pages", "head_dim", 0, A.EINVAL), ("pages", "dtype", 2, A.EUNSUPPORTED),
    ("pages", "dtype", -1, A.EUNSUPPORTED), ("pages", "n_pages", 1 << 27, A.EUNSUPPORTED), ("pages", "k", ADDR + 8, A.EINVAL),
    ("pages", "v", ADDR + 2, A.EINVAL), ("batch", "batch", 0, A.EINVAL), ("batch", "batch", 65536, A.EUNSUPPORTED),
    ("batch", "n_tokens", -1, A.EINVAL), ("batch", "max_q", -1, A.EINVAL), ("batch", "max_q", 11, A.EINVAL), ("batch", "max_kv", -1, A.EINVAL),
    ("batch", "max_kv", 65, A.EINVAL), ("batch", "table_width", 0, A.EINVAL), ("batch", "cu_q", None, A.EINVAL),
    ("batch", "kv_len", None, A.EINVAL), ("batch", "table", None, A.EINVAL), ("pages", "pos", ADDR + 4, A.EINVAL),
    ("pages", "weight", ADDR + 4, A.EINVAL), ("batch", "batch", 65535, A.OK),
])
def test_pages_and_batch_are_checked(name, where, field, value, code):
    pages, batch, rows, rot, sc = _args()
    if code == A.OK:                                   # the limit itself, in the one call that launches nothing
        name = "workspace"
    setattr(pages if where == "pages" else batch, field, value)
    assert _call(name, pages, batch, rows, rot, sc) == code


def test_sizes_whose_launches_would_be_too_large():
    pages, batch, rows, rot, sc = _args()
    batch.batch, pages.n_kv_heads = 32768, 33          # more than 2^20 sequences times heads
    assert _call("workspace", pages, batch, rows, rot, sc, hq=33) == A.EUNSUPPORTED
    pages.n_kv_heads, batch.max_kv, batch.table_width = 32, (1 << 20) + 1, (1 << 16) + 1
    assert _call("workspace", pages, batch, rows, rot, sc, hq=32) == A.EUNSUPPORTED
    pages, batch, rows, rot, sc = _args()
    batch.n_tokens = 1 << 27
    assert _call("workspace", pages, batch, rows, rot, sc, hq=16) == A.EUNSUPPORTED


@pytest.mark.parametrize("field,value", [("p", None), ("p", ADDR + 2), ("token_stride", 511), ("token_stride", -512), ("head_stride", 4),
                                         ("head_stride", -64)])
@pytest.mark.parametrize("name", ["append", "attention", "weights"])
def test_rows_are_checked(name, field, value):
    pages, batch, rows, rot, sc = _args()
    setattr(rows, field, value)
    assert _call(name, pages, batch, rows, rot, sc) == A.EINVAL


@pytest.mark.parametrize("name", ["workspace", "attention", "weights"])
def test_heads_are_checked(name):
    a = _args()
    assert _call(name, *a, hq=7) == A.EINVAL and _call(name, *a, hq=0) == A.EINVAL and _call(name, *a, hq=-2) == A.EINVAL
    assert _call(name, *a, hq=34) == A.EUNSUPPORTED       # 17 query heads per kv-head


@pytest.mark.parametrize("field,value", [("rot_dim", 8), ("rot_dim", -16), ("rot_dim", 80), ("n_axes", 0), ("n_axes", 5), ("adjacent", 2),
                                         ("freq", None)])
def test_rotary_is_checked(field, value):
    pages, batch, rows, rot, sc = _args()
    setattr(rot, field, value)
    assert _call("append", pages, batch, rows, rot, sc) == A.EINVAL


def test_append_refusals():
    pages, batch, rows, rot, sc = _args()
    rot.axis[31] = 1
    assert _call("append", pages, batch, rows, rot, sc) == A.EINVAL
    rot.axis[31] = 0
    assert _call("append", pages, batch, rows, rot, sc, positions=None) == A.EINVAL
    assert _call("append", pages, batch, rows, rot, sc, out=None) == A.EINVAL          # q without q_out
    assert _call("append", pages, batch, rows, rot, sc, out=ADDR + 4) == A.EINVAL
    assert _call("append", pages, batch, rows, rot, sc, hq=0) == A.EINVAL
    assert P.load().arkv_paged_append(None, None, None, 8, None, None, None, None, None, None) == A.EINVAL


@pytest.mark.parametrize("name", ["attention", "weights"])
def test_scores_are_checked(name):
    for field, value in [("scale", float("nan")), ("scale", float("inf")), ("cap", -1.0), ("cap", float("nan")), ("cap", float("inf")),
                         ("slopes", ADDR)]:                # slopes without q_pos
        pages, batch, rows, rot, sc = _args()
        setattr(sc, field, value)
        assert _call(name, pages, batch, rows, rot, sc) == A.EINVAL, field


def test_attention_and_weights_refusals():
    a = _args()
    assert _call("attention", *a, out=None) == A.EINVAL and _call("attention", *a, out=ADDR + 8) == A.EINVAL
    assert _call("weights", *a, lse=None) == A.EINVAL and _call("weights", *a, decay=float("nan")) == A.EINVAL
    a[0].weight = None
    assert _call("weights", *a) == A.EINVAL and _call("evict", *a) == A.EINVAL


def test_workspaces_that_are_too_small_are_refused():
    pages, batch, rows, rot, sc = _args()
    n = C.c_size_t()
    lib = P.load()
    assert lib.arkv_paged_workspace(C.byref(pages), C.byref(batch), 8, None) == A.EINVAL
    assert lib.arkv_paged_workspace(C.byref(pages), C.byref(batch), 8, C.byref(n)) == A.OK
    if n.value:
        for name in ("attention", "weights"):
            assert _call(name, pages, batch, rows, rot, sc, ws=None) == A.EINVAL
            assert _call(name, pages, batch, rows, rot, sc, size=n.value - 1) == A.EINVAL
            assert _call(name, pages, batch, rows, rot, sc, ws=ADDR + 4) == A.EINVAL


def test_a_batch_without_new_tokens():
    """Token-major arrays of no rows have no address: that is no error."""
    pages, batch, rows, rot, sc = _args()
    rows.p = None
    assert _call("append", pages, batch, rows, rot, sc) == A.EINVAL and _call("attention", pages, batch, rows, rot, sc) == A.EINVAL
    batch.n_tokens = batch.max_q = 0
    assert _call("append", pages, batch, rows, rot, sc, positions=None, out=None) == A.OK
    assert _call("attention", pages, batch, rows, rot, sc, out=None) == A.OK
    rows.token_stride = 4
    assert _call("append", pages, batch, rows, rot, sc) == A.EINVAL and _call("attention", pages, batch, rows, rot, sc) == A.EINVAL


def test_evictions_that_need_a_workspace():
    a = _args()
    a[1].table_width, a[1].max_kv = 4096, 36864
    for kw in [dict(max_keep=513, dst_width=33), dict(max_keep=32)]:   # more survivors, or more rows, than one workgroup takes
        assert _call("evict", *a, ws=None, **kw) == A.EINVAL
        assert _call("evict", *a, size=1 << 16, **kw) == A.EINVAL
        assert _call("evict", *a, ws=ADDR + 4, **kw) == A.EINVAL
        a[1].max_kv = 36865
    n = C.c_size_t()
    assert P.load().arkv_paged_workspace(C.byref(a[0]), C.byref(a[1]), 8, C.byref(n)) == A.OK and n.value > 1 << 16


def test_evict_refusals():
    a = _args()
    for kw in [dict(keep=None), dict(dst=None), dict(kept=None), dict(new_len=None), dict(max_keep=0), dict(max_keep=33), dict(sink=-1),
               dict(recent=-1), dict(dst_width=0)]:
        assert _call("evict", *a, **kw) == A.EINVAL, kw


def test_the_binding_takes_gpu_tensors_of_the_right_kind():
    z = torch.zeros
    with pytest.raises(ValueError):
        P.arkv_pages(z(4, 2, 16, 64, dtype=torch.bfloat16), z(4, 2, 16, 64, dtype=torch.bfloat16), z(4, 2, 16, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.arkv_pages(z(4, 2, 16, 64), z(4, 2, 16, 64), z(4, 2, 16, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.arkv_page_batch(z(3, dtype=torch.int32), z(2, dtype=torch.int32), z(2, 4, dtype=torch.int32), 4, 1, 64)
    with pytest.raises(ValueError):
        P.arkv_page_batch(z(3, dtype=torch.int32), z(2, dtype=torch.int32), z(2, 4, dtype=torch.int32), 4)
    with pytest.raises(ValueError):
        P.arkv_rotary(z(32, dtype=torch.float64))


def test_evictions_into_their_own_lengths_and_tables_are_refused():
    """Workgroups read kv_len, keep and the tables while others store kept and new_len."""
    # B = 2, 2 heads: kv_len and keep 8 bytes each, table 32, dst_table 16, kept [2][2][32] 512, new_len 8
    lengths, keep, table, dst, kept, new_len = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000
    for bad in [dict(new_len=lengths), dict(new_len=lengths + 4), dict(new_len=lengths - 4), dict(new_len=keep), dict(new_len=table + 28),
                dict(new_len=dst + 12), dict(kept=lengths), dict(kept=lengths - 508), dict(kept=keep + 4), dict(kept=table - 508),
                dict(kept=dst), dict(kept=new_len), dict(kept=new_len - 508), dict(new_len=kept + 508)]:
        a = _args()
        a[1].kv_len, a[1].table = lengths, table
        kw = dict(keep=keep, dst=dst, kept=kept, new_len=new_len)
        kw.update(bad)
        assert _call("evict", *a, **kw) == A.EINVAL, bad


def _size(hq, hkv, d, batch, n_tokens, max_q, max_kv):
    n = C.c_size_t()
    pages = P._Pages(0, 100, 64, hkv, d, ADDR, ADDR, ADDR, ADDR)
    b = P._Batch(batch, n_tokens, max_q, max_kv, 1 << 20, ADDR, ADDR, ADDR)
    assert P.load().arkv_paged_workspace(C.byref(pages), C.byref(b), hq, C.byref(n)) == A.OK
    return n.value


@pytest.mark.parametrize("large,small", [
    ((32, 32 * 2048, 2048, 16384), (32, 32, 1, 16384)), ((32, 32 * 2048, 2048, 16384), (1, 2048, 2048, 16384)),
    ((32, 32 * 2048, 2048, 16384), (1, 128, 128, 16384)), ((64, 64, 1, 4096), (1, 1, 1, 4096)), ((200, 200, 1, 30000), (2, 2, 1, 30000))])
def test_a_workspace_for_the_largest_batch_serves_smaller_ones(large, small):
    """Fewer rows are cut finer: the size must not go by the batch's own cut alone."""
    assert _size(32, 8, 128, *small) <= _size(32, 8, 128, *large)


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64), (16, 1, 128), (21, 3, 64), (64, 4, 128)])
def test_workspaces_grow_with_each_bound(hq, hkv, d):
    rng = np.random.default_rng(hq + d)
    for _ in range(3000):
        batch, n_tokens, max_kv = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (2000, 100000, 1 << 20))
        max_q = min(n_tokens, int(np.exp(rng.uniform(0, np.log(n_tokens + 1)))))
        more = [x + int(rng.integers(0, 3)) * int(rng.integers(0, x + 2)) for x in (batch, n_tokens, max_q, max_kv)]
        more[2] = min(more[2], more[1])
        a, b = _size(hq, hkv, d, batch, n_tokens, max_q, max_kv), _size(hq, hkv, d, *more)
        assert a <= b, (batch, n_tokens, max_q, max_kv, more)
        few = [max(1, int(x * rng.uniform())) for x in (batch, n_tokens, max_q, max_kv)]
        few[2] = min(few[2], few[1])
        assert _size(hq, hkv, d, *few) <= a, (batch, n_tokens, max_q, max_kv, few)


@pytest.mark.parametrize("batch,hkv,hq,max_q,n_tokens,max_kv", [
    (4096, 8, 8, 1, 4096, 1 << 20), (1024, 32, 32, 1, 1024, 1 << 20), (4096, 64, 64, 2, 8191, 1 << 18),
    (65535, 1, 16, 2000, 1 << 27, 128)])
def test_launches_that_cannot_be_made_are_refused_before_the_first(batch, hkv, hq, max_q, n_tokens, max_kv):
    """2^32 work-items or more, within every other bound: of the attention's launch, not of the joining one behind it."""
    pages, b, rows, rot, sc = _args()
    pages.n_kv_heads, b.batch, b.n_tokens, b.max_q, b.max_kv, b.table_width = hkv, batch, n_tokens, max_q, max_kv, 1 << 16
    if hq * n_tokens >= 1 << 31:                       # (that many tokens only without query heads)
        pages.n_pages = 1
        assert P.load().arkv_paged_append(C.byref(pages), C.byref(b), C.byref(rot), 0, None, C.byref(rows), C.byref(rows), ADDR, None, None) == A.EUNSUPPORTED
    else:
        assert _call("attention", pages, b, rows, rot, sc, hq=hq, size=1 << 50) == A.EUNSUPPORTED


def test_numbers_that_do_not_fit_32_bits_are_refused():
    """ctypes passes on the lowest 32 bits of a number: 2^32 + 64 rows would be 64."""
    big, z = (1 << 32) + 64, torch.zeros
    cu, lens, table = z(3, dtype=torch.int32), z(2, dtype=torch.int32), z(2, 4, dtype=torch.int32)
    for kw in [dict(n_tokens=big, max_q=1, max_kv=64), dict(n_tokens=4, max_q=big, max_kv=64), dict(n_tokens=4, max_q=1, max_kv=big),
               dict(n_tokens=4, max_q=1, page_size=1 << 30)]:
        with pytest.raises(ValueError, match="32 bits"):
            P.arkv_page_batch(cu, lens, table, **kw)
    with pytest.raises(ValueError, match="32 bits"):
        P.arkv_rotary(None, n_axes=(1 << 32) + 1)
    kw = dict(n_pages=4, page_size=16, n_kv_heads=1, kv_head=0, length=64, slot=0)
    for name in kw:
        with pytest.raises(ValueError, match="32 bits"):
            P.arkv_debug_paged_row(np.zeros(4, np.int32), **{**kw, name: kw[name] + (1 << 32)})


@pytest.mark.parametrize("budget", [0, -1, 65])
def test_the_example_refuses_budgets_that_no_cut_can_meet(budget):
    """With a budget above the limit a request would count rows that it never had."""
    from paper_2603_08727_amd.paged_example import PagedLayer
    with pytest.raises(ValueError, match="budget"):
        PagedLayer(1, limit=64, budget=budget, device="cpu")


@pytest.mark.parametrize("token_stride,head_stride", [(768, 64), (512, 128), (256, 64), (512, 0)])
def test_appends_in_place_of_rows_that_are_not_dense_are_refused(token_stride, head_stride):
    """Stored rows would lie over rows that are still to be read."""
    pages, batch, rows, rot, sc = _args()
    kv, q = P._Rows(0x100000, 128, 64), P._Rows(0x200000, token_stride, head_stride)
    assert P.load().arkv_paged_append(C.byref(pages), C.byref(batch), C.byref(rot), 8, C.byref(q), C.byref(kv), C.byref(kv), ADDR, 0x200000,
                                      None) == A.EINVAL
