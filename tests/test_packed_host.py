"""CPU checks of packed pages' and limited sight's entry points: refusals before anything is launched; and of the tests' own
plain forms."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2603_08727_amd import binding as A
from paper_2603_08727_amd import paged as P
import packed_ref as K

ADDR = 0x1000                                          # never followed: the calls are refused on the host


def _args(bits=8):
    packed = P._Packed(0, bits, 100, 16, 2, 64, ADDR, ADDR, ADDR, ADDR, ADDR)
    batch = P._Batch(2, 10, 5, 64, 4, ADDR, ADDR, ADDR)
    rows = P._Rows(ADDR, 512, 64)
    rot = P._Rotary(64, 1, 0, (C.c_uint8 * 64)(), ADDR)
    sc = P._Scores(0.125, 0.0, None, None, None)
    return packed, batch, rows, rot, sc


def _call(name, pages, batch, rows, rot, sc, hq=8, ws=ADDR, size=1 << 40, sight=None, **kw):
    lib, r = P.load(), C.byref
    if name == "append":
        return lib.arkv_packed_append(r(pages), r(batch), r(rot), hq, r(rows), r(rows), r(rows), kw.get("positions", ADDR), kw.get("out", ADDR), None)
    if name == "read":
        return lib.arkv_packed_read(r(pages), r(batch), kw.get("out", ADDR), kw.get("out", ADDR), None)
    if name == "workspace":
        return lib.arkv_packed_workspace(r(pages), r(batch), hq, r(C.c_size_t()))
    if name == "sight":
        plain = P._Pages(0, pages.n_pages, pages.page_size, pages.n_kv_heads, pages.head_dim, pages.k, pages.v, pages.pos, None)
        return lib.arkv_paged_attention_sight(r(plain), r(batch), r(sc), sight if sight is None else r(sight), hq, r(rows), kw.get("out", ADDR), None, ws,
                                              size, None)
    return lib.arkv_packed_attention(r(pages), r(batch), r(sc), sight if sight is None else r(sight), hq, r(rows), kw.get("out", ADDR), None, ws, size, None)


@pytest.mark.parametrize("name", ["append", "read", "workspace", "attention"])
@pytest.mark.parametrize("where,field,value,code", [
    ("pages", "k", None, A.EINVAL), ("pages", "v", None, A.EINVAL), ("pages", "pos", None, A.EINVAL), ("pages", "k_scale", None, A.EINVAL),
    ("pages", "v_scale", None, A.EINVAL), ("pages", "k_scale", ADDR + 8, A.EINVAL), ("pages", "v_scale", ADDR + 2, A.EINVAL),
    ("pages", "k", ADDR + 8, A.EINVAL), ("pages", "v", ADDR + 4, A.EINVAL), ("pages", "bits", 16, A.EUNSUPPORTED), ("pages", "bits", 0, A.EUNSUPPORTED),
    ("pages", "bits", 2, A.EUNSUPPORTED), ("pages", "n_pages", 0, A.EINVAL), ("pages", "n_pages", 1 << 27, A.EUNSUPPORTED),
    ("pages", "page_size", 24, A.EINVAL), ("pages", "page_size", 8, A.EUNSUPPORTED), ("pages", "page_size", 2048, A.EUNSUPPORTED),
    ("pages", "head_dim", 32, A.EUNSUPPORTED), ("pages", "dtype", 2, A.EUNSUPPORTED), ("batch", "batch", 0, A.EINVAL),
    ("batch", "n_tokens", -1, A.EINVAL), ("batch", "max_q", 11, A.EINVAL), ("batch", "max_kv", 65, A.EINVAL), ("batch", "cu_q", None, A.EINVAL),
    ("batch", "kv_len", None, A.EINVAL), ("batch", "table", None, A.EINVAL)])
def test_packed_pages_and_batch_are_checked(name, where, field, value, code):
    a = _args()
    setattr(a[0] if where == "pages" else a[1], field, value)
    assert _call(name, *a) == code


def test_refusals_of_append_and_read():
    a = _args(4)
    a[3].axis[31] = 1
    assert _call("append", *a) == A.EINVAL
    a = _args(4)
    assert _call("append", *a, positions=None) == A.EINVAL and _call("append", *a, out=None) == A.EINVAL
    assert _call("append", *a, out=ADDR + 4) == A.EINVAL and _call("append", *a, hq=0) == A.EINVAL
    assert _call("read", *a, out=ADDR + 8) == A.EINVAL
    assert _call("read", *a, out=None) == A.OK         # nothing is wanted
    for field, value in [("rot_dim", 8), ("rot_dim", 80), ("n_axes", 0), ("adjacent", 2), ("freq", None)]:
        a = _args()
        setattr(a[3], field, value)
        assert _call("append", *a) == A.EINVAL
    a = _args()
    a[1].n_tokens = a[1].max_q = 0
    assert _call("append", *a, positions=None, out=None) == A.OK and _call("read", *a) == A.OK
    assert P.load().arkv_packed_append(None, None, None, 8, None, None, None, None, None, None) == A.EINVAL
    assert P.load().arkv_packed_read(None, None, None, None, None) == A.EINVAL


@pytest.mark.parametrize("name", ["attention", "sight"])
def test_refusals_of_attention(name):
    a = _args()
    s = P._Sight(16, 4, 0, None)
    assert _call(name, *a, sight=s, out=None) == A.EINVAL and _call(name, *a, sight=s, out=ADDR + 8) == A.EINVAL
    assert _call(name, *a, sight=s, hq=7) == A.EINVAL and _call(name, *a, sight=s, hq=34) == A.EUNSUPPORTED
    assert _call(name, *a, sight=s, ws=None) == A.EINVAL and _call(name, *a, sight=s, ws=ADDR + 4) == A.EINVAL
    assert _call(name, *a, sight=s, size=(1 << 16) - 1) == A.EINVAL
    for bad in [P._Sight(-1, 0, 0, None), P._Sight(0, -1, 0, None), P._Sight(16, -4, 0, None), P._Sight(0, 0, 0, ADDR), P._Sight(0, 0, -1, ADDR),
                P._Sight(0, 0, 1, ADDR + 4), P._Sight(8, 0, 0, ADDR)]:
        assert _call(name, *a, sight=bad) == A.EINVAL, (bad.window, bad.sink, bad.tree_words, bad.tree)
    a[1].n_tokens, a[1].max_q = 200, 65                # 65 new tokens need two words
    assert _call(name, *a, sight=P._Sight(0, 0, 1, ADDR)) == A.EINVAL
    a = _args()
    a[4].slopes = ADDR                                 # slopes without q_pos
    assert _call(name, *a, sight=s) == A.EINVAL
    a = _args()
    a[2].head_stride = 4
    assert _call(name, *a, sight=s) == A.EINVAL
    a = _args()
    a[1].n_tokens = a[1].max_q = 0
    a[2].p = None
    assert _call(name, *a, sight=s, out=None) == A.OK


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64), (16, 1, 128), (21, 3, 64)])
def test_a_workspace_serves_every_window(hq, hkv, d):
    """A window shortens the sequences, so that their keys are cut finer: no call may need more than the workspace's size."""
    rng = np.random.default_rng(hq + d)
    lib, n = P.load(), C.c_size_t()
    plain = P._Pages(0, 100, 64, hkv, d, ADDR, ADDR, ADDR, ADDR)
    packed = P._Packed(0, 8, 100, 64, hkv, d, ADDR, ADDR, ADDR, ADDR, ADDR)
    rows, sc = P._Rows(ADDR, hq * d, d), P._Scores(0.125, 0.0, None, None, None)
    for _ in range(1500):
        batch, n_tokens, max_kv, window, sink = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (500, 30000, 1 << 20, 1 << 20, 1000))
        max_q = min(n_tokens, int(np.exp(rng.uniform(0, np.log(n_tokens + 1)))))
        b = P._Batch(batch, n_tokens, max_q, max_kv, 1 << 20, ADDR, ADDR, ADDR)
        for pages, size, call in ((plain, lib.arkv_paged_workspace, lib.arkv_paged_attention_sight), (packed, lib.arkv_packed_workspace, lib.arkv_packed_attention)):
            assert size(C.byref(pages), C.byref(b), hq, C.byref(n)) == A.OK
            # (refused for its output alone, which is checked behind the workspace: with one that is too small too)
            for s in (None, P._Sight(window, sink, 0, None), P._Sight(window, sink, 1 << 10, ADDR)):
                args = (C.byref(pages), C.byref(b), C.byref(sc), s if s is None else C.byref(s), hq, C.byref(rows))
                assert call(*args, ADDR, None, ADDR, 0, None) == A.EINVAL
                need = _need(call, args, n.value)
                assert need <= n.value, (batch, n_tokens, max_q, max_kv, window, sink)


def _need(call, args, most):
    """Whether a workspace of `most` bytes is taken: without a GPU a call that passes its checks fails in the launch."""
    if torch.cuda.is_available():
        pytest.skip("would launch")
    rc = call(*args, ADDR, None, ADDR, most, None)
    return most if rc in (A.EHIP, A.EUNSUPPORTED) else most + 1


def test_the_binding_checks_packed_pages_and_sights():
    z, u8, i32 = torch.zeros, torch.uint8, torch.int32
    with pytest.raises(ValueError):                    # on the CPU
        P.arkv_packed_pages(z(4, 2, 16, 64, dtype=u8), z(4, 2, 16, 64, dtype=u8), z(4, 2, 16, 2, dtype=u8), z(4, 2, 16, 2, dtype=u8), z(4, 2, 16, dtype=i32),
                            torch.bfloat16)
    with pytest.raises(ValueError, match="bits"):      # 96 bytes of 64 channels
        P.arkv_packed_pages(z(4, 2, 16, 96, dtype=u8), z(4, 2, 16, 96, dtype=u8), z(4, 2, 16, 2, dtype=u8), z(4, 2, 16, 2, dtype=u8), z(4, 2, 16, dtype=i32),
                            torch.bfloat16)
    with pytest.raises(ValueError, match="dtype"):
        P.arkv_packed_pages(z(4, 2, 16, 64, dtype=u8), z(4, 2, 16, 64, dtype=u8), z(4, 2, 16, 2, dtype=u8), z(4, 2, 16, 2, dtype=u8), z(4, 2, 16, dtype=i32),
                            torch.float32)
    for kw in [dict(window=1 << 32), dict(sink=1 << 31)]:
        with pytest.raises(ValueError, match="32 bits"):
            P.arkv_sight(**kw)
    with pytest.raises(ValueError, match="word"):
        P.arkv_sight(tree=z(4, 0, dtype=torch.int64))
    for tree in [z(4, 1), z(4, dtype=torch.int64), z(4, 1, dtype=i32), z(4, 1, dtype=torch.int64)]:     # (the last: on the CPU)
        with pytest.raises(ValueError):
            P.arkv_sight(tree=tree)


# ---- the plain forms themselves -------------------------------------------------------------------

@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_packing_by_the_book(bits, dtype):
    top = K.FORMS[bits][2]
    g = torch.Generator().manual_seed(bits)
    x = (torch.randn(40, 32, generator=g) * 2.0 ** torch.randint(-10, 6, (40, 1), generator=g)).to(dtype).double()
    codes, scale = K.pack(x, bits, dtype)
    y = K.values(codes, scale, bits)
    unit = torch.ldexp(torch.ones(40, 1, dtype=torch.float64), scale.int() - 127)
    assert (x.abs().amax(1, keepdim=True) <= top * unit).all() and (x.abs().amax(1, keepdim=True) > top / 2 * unit).all()
    step = torch.where((y / unit).abs() < 2.0 ** (-6 if bits == 8 else 0), torch.tensor(2.0 ** (-9 if bits == 8 else -1), dtype=torch.float64),
                       torch.ldexp(torch.ones_like(y), torch.frexp((y / unit).abs())[1] - 1 - K.FORMS[bits][1])) * unit
    assert ((x - y).abs() <= step / 2).all()
    again = K.pack(y, bits, dtype)
    assert torch.equal(K.values(*again, bits), y)
    if bits == 8:
        assert torch.equal((x / unit).float().to(torch.float8_e4m3fn).double() * unit, y)


@pytest.mark.parametrize("bits", [8, 4])
def test_packing_at_the_borders(bits):
    ties = (K.table(bits)[:7] + K.table(bits)[1:8]) / 2
    x = torch.zeros(5, 32, dtype=torch.float64)
    x[0, :7], x[0, 31] = ties, K.FORMS[bits][2]
    x[1, 0], x[2, :2], x[3, 5] = -0.0, torch.tensor([math.nan, 1.0]), math.inf
    x[4, 0] = float(torch.finfo(torch.bfloat16).max)
    codes, scale = K.pack(x, bits, torch.bfloat16)
    full = codes if bits == 8 else torch.stack([codes & 15, codes >> 4], -1).reshape(5, 32)
    assert full[0, :7].tolist() == [0, 2, 2, 4, 4, 6, 6] and scale[0, 0] == 127 and scale[1, 0] == 1 and full[1, 0] == 1 << bits - 1
    assert (scale[2, 0] == 255) == (bits == 4) and (bits == 4 or full[2, 0] == 127 and full[3, 5] == 127)
    assert K.values(codes, scale, bits)[4, 0] == (240.0 if bits == 8 else 3.0) * 2.0 ** (120 if bits == 8 else 126)


def test_sights_by_the_book():
    from types import SimpleNamespace
    s = SimpleNamespace(q_len=[3], kv_len_list=[8], table=torch.zeros(1, 1, dtype=torch.int32), pos=torch.zeros(1, 1, 16, dtype=torch.int32), page=16, n_pages=1)
    see = lambda **kw: [[j for j in range(8) if x[j]] for x in K.sight(s, 0, **kw).tolist()]  # noqa: E731
    assert see() == [list(range(6)), list(range(7)), list(range(8))]
    assert see(window=2) == [[4, 5], [5, 6], [6, 7]] and see(window=2, sink=1) == [[0, 4, 5], [0, 5, 6], [0, 6, 7]]
    tree = torch.tensor([[1, 0, 0], [1, 1, 0], [1, 0, 1]], dtype=torch.bool)
    assert see(tree=tree) == [[0, 1, 2, 3, 4, 5], [0, 1, 2, 3, 4, 5, 6], [0, 1, 2, 3, 4, 5, 7]]
    assert see(tree=tree, window=3) == [[3, 4, 5], [4, 5, 6], [4, 5, 7]]
    assert see(window=1, prefix=[3]) == [[0, 1, 2, 5], [0, 1, 2, 6], [0, 1, 2, 7]]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_every_pair_of_code_and_scale_is_there(bits, d):
    codes, scale = K.every_pair(bits, d)
    assert len(codes) == len(scale)
    pairs = {(int(s), int(c)) for row, of in zip(codes, scale) for c, s in zip(row, of.repeat_interleave(32 * bits // 8))}
    assert pairs == {(s, c) for s in range(256) for c in range(256)}


@pytest.mark.parametrize("hkv", [2, 64, 128])
def test_each_entry_point_takes_its_own_kind_of_pages(hkv):
    """A struct of the other kind would be read with its fields moved: 64 kv-heads as 64 channels, the scale bytes as weights."""
    batch = P._Batch(2, 10, 5, 64, 4, ADDR, ADDR, ADDR)
    packed = P._Packed(0, 8, 64, 16, hkv, 64, ADDR, ADDR, ADDR, ADDR, ADDR)
    plain = P._Pages(0, 64, 16, hkv, 64, ADDR, ADDR, ADDR, ADDR)

    class Held:
        def __init__(self, c):
            self.c, self.ref, self.index, self.device = c, C.addressof(c), 0, "cuda:0"

    def kind(cls, c):
        x = cls.__new__(cls)
        Held.__init__(x, c)
        return x

    b, pk, pl = Held(batch), kind(P.arkv_packed_pages, packed), kind(P.arkv_pages, plain)
    for call in [lambda: P.arkv_paged_workspace_bytes(pk, b, 2 * hkv), lambda: P.arkv_paged_workspace(pk, b, 2 * hkv),
                 lambda: P.arkv_paged_append(pk, b, None, None, None, None, None, None), lambda: P.arkv_paged_attention(pk, b, None, 1.0, None),
                 lambda: P.arkv_paged_attention_sight(pk, b, None, None, 1.0, None), lambda: P.arkv_paged_weights(pk, b, None, 1.0, None),
                 lambda: P.arkv_paged_evict(pk, b, None, None, None, None),
                 lambda: P.arkv_packed_workspace_bytes(pl, b, 2 * hkv), lambda: P.arkv_packed_workspace(pl, b, 2 * hkv),
                 lambda: P.arkv_packed_append(pl, b, None, None, None, None, None, None), lambda: P.arkv_packed_read(pl, b, None, None),
                 lambda: P.arkv_packed_attention(pl, b, None, 1.0, None)]:
        with pytest.raises(ValueError, match="pages: expected"):
            call()
    assert P.arkv_packed_workspace_bytes(pk, b, 2 * hkv) >= 1 << 16 and P.arkv_paged_workspace_bytes(pl, b, 2 * hkv) >= 1 << 16
