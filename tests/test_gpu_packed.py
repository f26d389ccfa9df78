"""GPU tests of packed pages, and of attention under a window or over drafted trees, against plain 64-bit forms
(tests/packed_ref.py)."""
import math

import pytest
import torch

from paper_2603_08727_amd import paged as P
import packed_ref as K
import paged_ref as R

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
TICKETS = 1 << 16                                      # bytes of a workspace that are zero between calls


def handles(s, max_q=None, max_kv=None):
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, s.max_q if max_q is None else max_q, s.max_kv if max_kv is None else max_kv)
    if hasattr(s, "bits"):
        pages = P.arkv_packed_pages(s.k_codes, s.v_codes, s.k_scale, s.v_scale, s.pos, s.dtype)
        return pages, batch, P.arkv_packed_workspace(pages, batch, s.hq)
    pages = P.arkv_pages(s.k, s.v, s.pos)
    return pages, batch, P.arkv_paged_workspace(pages, batch, s.hq)


def attend(s, window=0, sink=0, tree=None, ws=None, **kw):
    pages, batch, own = handles(s)
    ws = own if ws is None else ws
    ws[TICKETS:].fill_(0xFF)                           # what a workspace holds behind its tickets does not matter
    out = torch.full((s.n, s.hq, s.d), 7.0, dtype=s.dtype, device="cuda")
    lse = torch.full((s.n, s.hq), 7.0, device="cuda")
    sight = None
    if window or sink or tree is not None:
        sight = P.arkv_sight(window, sink, None if tree is None else K.words(tree).cuda())
    if hasattr(s, "bits"):
        P.arkv_packed_attention(pages, batch, s.q, s.scale, out, lse=lse, sight=sight, workspace=ws, **kw)
    else:
        P.arkv_paged_attention_sight(pages, batch, sight, s.q, s.scale, out, lse=lse, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert not ws[:TICKETS].any()
    return out, lse


def check(s, window=0, sink=0, tree=None, **kw):
    out, lse = attend(s, window, sink, tree, **kw)
    ref, rl, tol, ltol = K.attention(s, window, sink, tree, **kw)
    n = sum(s.q_len)
    R.close(out[:n], ref[:n], tol[:n], "out")
    R.close(lse[:n], rl[:n], ltol[:n], "lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()      # rows of no sequence are left alone
    return out, lse


def slopes_of(s):
    sl = 2.0 ** (-8.0 * (torch.arange(s.hq, device="cuda", dtype=torch.float32) + 1) / s.hq)
    qp = torch.cat([torch.arange(t - a, t, device="cuda", dtype=torch.int32) * 2 + 1 for a, t in zip(s.q_len, s.kv_len_list)] +
                   [torch.zeros(s.n - sum(s.q_len), device="cuda", dtype=torch.int32)])
    return sl, qp


def scores_of(kind, s, q, kv):
    kw = {}
    if "cap" in kind:
        kw["cap"] = 3.5
    if "distance" in kind:
        kw["slopes"], kw["q_pos"] = slopes_of(s)
    if "prefix" in kind:
        pre = [min(t, t - a + (2 * a) // 3) for a, t in zip(q, kv)]
        pre[0] = min(9, kv[0])
        if len(pre) > 1:
            pre[1] = -4
        kw["prefix"] = torch.tensor(pre, dtype=torch.int32, device="cuda")
    return kw


# ---- packed rows ----------------------------------------------------------------------------------

def pool(bits, n_pages, hkv, page, d, dtype, fill=0xA5):
    new = lambda *shape: torch.full(shape, fill, dtype=torch.uint8, device="cuda")  # noqa: E731
    pos = torch.full((n_pages, hkv, page), -3, dtype=torch.int32, device="cuda")
    return P.arkv_packed_pages(new(n_pages, hkv, page, d * bits // 8), new(n_pages, hkv, page, d * bits // 8), new(n_pages, hkv, page, d // 32),
                               new(n_pages, hkv, page, d // 32), pos, dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [8, 4])
def test_every_code_and_scale_is_read_as_its_value(bits, d, dtype):
    """Any bytes are rows: codes and scales at random, every pair of them among them."""
    g = torch.Generator().manual_seed(d + bits)
    n_pages, hkv, page = 40, 3, 64
    pages = pool(bits, n_pages, hkv, page, d, dtype)
    for x in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        x.copy_(torch.randint(0, 256, x.shape, generator=g, dtype=torch.int32).to(torch.uint8))
    flat, scales = pages.k.view(-1, pages.k.shape[-1]), pages.k_scale.view(-1, d // 32)
    per = min(32 * bits // 8, 16)
    for i in range(0, 256, per):                       # row: one scale, `per` codes at a time
        row = torch.arange(256) + i // per * 256
        flat[row % len(flat), :per] = torch.arange(i, i + per, dtype=torch.int32).to(torch.uint8).cuda()
        scales[row % len(flat), 0] = torch.arange(256, dtype=torch.int32).to(torch.uint8).cuda()
    kv = [n_pages * page // 2 - 7, n_pages * page // 2]
    table = torch.full((2, n_pages // 2), -1, dtype=torch.int32)
    table[0], table[1] = torch.arange(n_pages // 2), torch.arange(n_pages // 2, n_pages)
    n = sum(kv)
    batch = P.arkv_page_batch(torch.tensor([0, kv[0], n], dtype=torch.int32).cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), table.cuda(), n, max(kv), max(kv))
    k, v = (torch.full((n, hkv, d), 7.0, dtype=dtype, device="cuda") for _ in "kv")
    P.arkv_packed_read(pages, batch, k, v)
    only = torch.full_like(v, 7.0)
    P.arkv_packed_read(pages, batch, None, only)
    torch.cuda.synchronize()
    for got, codes, scale in ((k, pages.k, pages.k_scale), (v, pages.v, pages.v_scale), (only, pages.v, pages.v_scale)):
        want = K.values(codes.cpu(), scale.cpu(), bits).transpose(1, 2).reshape(n_pages * page, hkv, d)
        want = torch.cat([want[:kv[0]], want[n_pages // 2 * page:]])
        want = want.float().to(dtype)                  # (codes' values fit 32 bits)
        got = got.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = ~torch.isnan(want)
        assert torch.equal(got[ok], want[ok])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [8, 4])
def test_every_pair_of_code_and_scale_is_read(bits, d, dtype):
    """All of them in rows of the batch: keys in order, values the other way round."""
    codes, scale = K.every_pair(bits, d)
    n, page = len(codes), 64
    pages = pool(bits, n // page, 1, page, d, dtype)
    for x, y in ((pages.k, codes), (pages.v, codes.flip(0)), (pages.k_scale, scale), (pages.v_scale, scale.flip(0))):
        x.copy_(y.reshape(x.shape))
    one = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = P.arkv_page_batch(one([0, n]), one([n]), one([list(range(n // page))]), n, n, n)
    k, v = (torch.full((n, 1, d), 7.0, dtype=dtype, device="cuda") for _ in "kv")
    P.arkv_packed_read(pages, batch, k, v)
    want = K.values(codes, scale, bits).float().to(dtype)              # (codes' values fit 32 bits)
    for got, ref in ((k, want), (v, want.flip(0))):
        got = got[:, 0].cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(got[~torch.isnan(ref)], ref[~torch.isnan(ref)])


def check_append(pages, batch, s, kn, vn, positions, rotary, freq, axis, adjacent, q=None, q_out=None):
    """Appends, and compares every byte of the pool."""
    before = [x.clone().cpu() for x in (pages.k, pages.v, pages.k_scale, pages.v_scale, pages.pos)]
    P.arkv_packed_append(pages, batch, rotary, q, kn, vn, positions, q_out)
    torch.cuda.synchronize()
    after = [x.cpu() for x in (pages.k, pages.v, pages.k_scale, pages.v_scale, pages.pos)]
    turned = kn.cpu().double()
    half = 0 if freq is None else freq.numel()
    for i in range(half):
        a, e = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        t = positions[axis[i]].cpu().double() * freq[i].cpu().double()
        c, sn = torch.cos(t)[:, None], torch.sin(t)[:, None]
        xa, xe = turned[..., a].clone(), turned[..., e].clone()
        turned[..., a], turned[..., e] = xa * c - xe * sn, xe * c + xa * sn
    kc, ks = K.pack(turned, pages.bits, pages.dtype)
    vc, vs = K.pack(vn.cpu().double(), pages.bits, pages.dtype)
    for b, (a, t) in enumerate(zip(s.q_len, s.kv_len_list)):
        at = sum(s.q_len[:b])
        for i in range(a):
            slot = t - a + i
            page = int(s.table[b, slot // s.page]) if slot >= 0 else -1
            if not 0 <= page < pages.n_pages:
                continue
            off, j = slot % s.page, at + i
            K.same_values(after[0][page, :, off], after[2][page, :, off], kc[j], ks[j], pages.bits)
            K.same_values(after[1][page, :, off], after[3][page, :, off], vc[j], vs[j], pages.bits)
            assert (after[4][page, :, off] == int(positions[0, j])).all()
            for x, y in zip(before, after):            # seen: the rest has to be as it was
                x[page, :, off] = y[page, :, off]
    assert all(torch.equal(x, y) for x, y in zip(before, after))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("bits,hq,hkv,d,axes,rot,adjacent", [
    (8, 8, 2, 64, 1, 64, False), (4, 8, 2, 128, 3, 128, False), (8, 12, 4, 128, 2, 64, True), (4, 3, 3, 64, 1, 32, False), (8, 5, 1, 128, 1, 0, False),
    (4, 16, 16, 128, 1, 128, True), (8, 4, 2, 64, 4, 16, False), (4, 6, 3, 64, 2, 48, True), (8, 2, 1, 128, 1, 80, False)])
@pytest.mark.parametrize("q,kv", [((1,), (1,)), ((1, 1, 0, 1), (17, 300, 5, 64)), ((70, 3, 1), (71, 90, 16))])
def test_append(q, kv, bits, hq, hkv, d, axes, rot, adjacent, dtype):
    s = R.problem("cuda", dtype, hq, hkv, d, 16, q, kv, seed=rot + hq, extra_tokens=2)
    pages = pool(bits, s.n_pages, hkv, 16, d, dtype)
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, s.max_q, s.max_kv)
    g = torch.Generator().manual_seed(5)
    qkv = (torch.randn(s.n, hq + 2 * hkv, d, generator=g) * 2.0 ** torch.randint(-6, 4, (s.n, 1, 1), generator=g)).to(dtype).cuda()
    qn, kn, vn = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    positions = torch.randint(0, 1 << 20, (axes, s.n), generator=g, dtype=torch.int32).cuda()
    freq = None if rot == 0 else (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).cuda()
    axis = [i % axes for i in range(rot // 2)]
    rotary = P.arkv_rotary(freq, axis, axes, adjacent)
    q_out, q_16 = (torch.full((s.n, hq, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    check_append(pages, batch, s, kn, vn, positions, rotary, freq, axis, adjacent, qn, q_out)
    plain = P.arkv_pages(torch.zeros_like(s.k), torch.zeros_like(s.v), torch.zeros_like(s.pos))
    P.arkv_paged_append(plain, batch, rotary, qn, kn, vn, positions, q_16)
    assert torch.equal(q_out, q_16)                    # queries are turned as on the way to 16-bit pages


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("bits", [8, 4])
def test_append_of_ties_zeros_limits_and_no_numbers(bits, dtype):
    s = R.problem("cuda", dtype, 1, 1, 64, 16, (40,), (48,), seed=1)
    pages = pool(bits, s.n_pages, 1, 16, 64, dtype)
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, s.max_q, s.max_kv)
    up, top = K.table(bits)[:1 << bits - 1], K.FORMS[bits][2]
    up = up[up <= top].float()
    ties = (up[1:] + up[:-1]) / 2
    x = torch.zeros(40, 64)
    for r in range(8):                                 # every tie, and its neighbours, under a scale that the block's last channel holds
        part = ties[8 * r:8 * r + 8] if bits == 8 else ties
        x[r, :len(part)], x[r, 8:8 + len(part)], x[r, 16:16 + len(part)], x[r, 31] = part, -part, part * (1 + 2.0 ** -7), top
        x[r, 32:32 + len(part)], x[r, 63] = part * (1 - 2.0 ** -7), -top
    for i, r in enumerate(range(8, 16)):               # just on and just over the largest value of a scale
        x[r, 0], x[r, 1], x[r, 32], x[r, 33] = top * 2.0 ** (i - 4), 1.0, top * 2.0 ** (i - 4) * (1 + 2.0 ** -7), -0.0
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    x[16, 0], x[17, 3], x[18, 0], x[19, :] = big, -big, big * (1 - 2.0 ** -5), big
    x[20, 0], x[21, :] = small, torch.linspace(-2 * small, 2 * small, 64)
    x[22, :] = torch.arange(64) * (2.0 ** -133 if dtype == BF else 2.0 ** -24)
    x[23, 5], x[24, 40], x[25, 7], x[26, :] = math.nan, math.inf, -math.inf, math.nan
    x[23, 6], x[24, 41], x[25, 1] = 3.0, -2.0, 500.0
    x = x.to(dtype).cuda()[:, None]
    check_append(pages, batch, s, x.contiguous(), x.flip(0).contiguous(), torch.zeros(1, 40, dtype=torch.int32, device="cuda"), P.arkv_rotary(None), None, [], False)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("bits", [8, 4])
def test_append_of_keys_that_leave_the_type_as_they_turn(bits, dtype):
    s = R.problem("cuda", dtype, 1, 1, 64, 16, (20,), (20,), seed=1)
    pages = pool(bits, s.n_pages, 1, 16, 64, dtype)
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, s.max_q, s.max_kv)
    g = torch.Generator().manual_seed(2)
    x = (torch.randn(20, 1, 64, generator=g) * torch.finfo(dtype).max).clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max).to(dtype).cuda()
    freq = (torch.rand(32, generator=g, dtype=torch.float64) * 3).cuda()
    rotary = P.arkv_rotary(freq)
    check_append(pages, batch, s, x, x, torch.arange(20, dtype=torch.int32, device="cuda")[None], rotary, freq, [0] * 32, False)


@pytest.mark.parametrize("bits", [8, 4])
def test_append_and_read_without_slots_pages_or_sequences(bits):
    s = R.problem("cuda", BF, 4, 2, 64, 16, (5, 20, 2), (3, 40, 30), seed=4, extra_tokens=3)
    s.table[1, 1], s.table[2, 1] = s.n_pages, -1
    pages = pool(bits, s.n_pages, 2, 16, 64, BF)
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, s.max_q, s.max_kv)
    g = torch.Generator().manual_seed(5)
    kn, vn = (torch.randn(s.n, 2, 64, generator=g).to(BF).cuda() for _ in "kv")
    positions = torch.arange(s.n, dtype=torch.int32, device="cuda")[None]
    freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).cuda()
    q = torch.randn(s.n, 4, 64, generator=g).to(BF).cuda()
    want = q.clone()
    check_append(pages, batch, s, kn, vn, positions, P.arkv_rotary(freq), freq, [0] * 32, False, q, q)      # in place
    plain = P.arkv_pages(torch.zeros_like(s.k), torch.zeros_like(s.v), torch.zeros_like(s.pos))
    P.arkv_paged_append(plain, batch, P.arkv_rotary(freq), want, kn, vn, positions, want)
    assert torch.equal(q, want)
    k, v = (torch.full((s.n, 2, 64), 7.0, dtype=BF, device="cuda") for _ in "kv")
    P.arkv_packed_read(pages, batch, k, v)
    torch.cuda.synchronize()
    there = [False] * 2 + [True] * 3 + [not 16 <= j < 32 for j in range(20, 40)] + [False, False]
    there = torch.tensor(there, device="cuda")
    n = sum(s.q_len)
    for x in (k, v):
        assert (x[n:] == 7).all() and (x[:n][~there] == 0).all() and (x[:n][there].abs().amax((1, 2)) > 0).all()


def test_rows_are_read_from_far_behind_4_gb():
    """One pool whose last rows lie beyond 2^32 bytes; keys and values share it."""
    n_pages, hkv, page, d = 70000, 8, 64, 128
    codes = torch.empty(n_pages, hkv, page, d, dtype=torch.uint8, device="cuda")
    scale = torch.empty(n_pages, hkv, page, 4, dtype=torch.uint8, device="cuda")
    pos = torch.empty(n_pages, hkv, page, dtype=torch.int32, device="cuda")
    assert codes.numel() > 1 << 32
    s = K.problem("cuda", 8, BF, hq=16, hkv=hkv, d=d, page=page, q_len=(3, 1, 70), kv_len=(200, 500, 300), seed=8)
    to = torch.arange(s.n_pages, device="cuda") * 11 + (n_pages - 11 * s.n_pages)
    codes[to], scale[to], pos[to] = s.k_codes, s.k_scale, s.pos
    far = K.problem("cuda", 8, BF, hq=16, hkv=hkv, d=d, page=page, q_len=(3, 1, 70), kv_len=(200, 500, 300), seed=8)
    far.v, far.v_codes, far.v_scale = s.k, s.k_codes, s.k_scale
    ref, rl, tol, ltol = K.attention(far)
    s.k_codes = s.v_codes = codes
    s.k_scale = s.v_scale = scale
    s.pos, s.n_pages = pos, n_pages
    s.table = torch.where(s.table >= 0, to[s.table.clamp(min=0).long()].int(), s.table)
    out, lse = attend(s)
    R.close(out, ref, tol, "out")
    R.close(lse, rl, ltol, "lse")
    k = torch.empty(s.n, hkv, d, dtype=BF, device="cuda")
    pages, batch, _ = handles(s)
    P.arkv_packed_read(pages, batch, k, None)
    rows = [R.rows(far, far.k, b, 0)[0][-a:] for b, a in enumerate(far.q_len)]
    assert torch.equal(k[:, 0], torch.cat(rows))
    # rows appended there, against a small pool's
    g = torch.Generator().manual_seed(1)
    kn, vn = (torch.randn(s.n, hkv, d, generator=g).to(BF).cuda() for _ in "kv")
    freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    positions = torch.arange(s.n, dtype=torch.int32, device="cuda")[None]
    scale_v, codes_v = torch.empty_like(scale), torch.empty_like(codes)
    there = P.arkv_packed_pages(codes, codes_v, scale, scale_v, pos, BF)
    near, near_batch, _ = handles(far)
    near = P.arkv_packed_pages(torch.zeros_like(far.k_codes), torch.zeros_like(far.k_codes), torch.zeros_like(far.k_scale), torch.zeros_like(far.k_scale),
                               torch.zeros_like(far.pos), BF)
    got = []
    for p, b in ((there, batch), (near, near_batch)):
        P.arkv_packed_append(p, b, P.arkv_rotary(freq), None, kn, vn, positions, None)
        read = [torch.empty(s.n, hkv, d, dtype=BF, device="cuda") for _ in "kv"]
        P.arkv_packed_read(p, b, *read)
        got.append(read)
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


# ---- attention over packed pages ------------------------------------------------------------------

STEPS = [((1,), (1,)), ((1,), (2,)), ((1,), (17,)), ((1, 1, 1), (63, 64, 65)), ((1, 1), (1000, 31)), ((1, 0, 1, 1), (129, 0, 513, 2)),
         ((1,) * 9, (5, 700, 33, 1, 2049, 64, 96, 128, 300))]
CHUNKS = [((2,), (2,)), ((16, 1), (16, 40)), ((17,), (17,)), ((33, 0, 5), (64, 0, 5)), ((64,), (1000,)), ((129, 1, 77), (300, 1025, 77)),
          ((300,), (2100,)), ((5, 1, 1, 40), (900, 3, 700, 41))]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("bits,hq,hkv,d,page", [(8, 8, 2, 64, 16), (4, 8, 2, 128, 32), (8, 3, 3, 128, 16), (4, 12, 4, 64, 64), (8, 16, 1, 128, 128),
                                                (4, 16, 1, 64, 16)])
@pytest.mark.parametrize("i", range(len(STEPS) + len(CHUNKS)))
def test_packed_attention(i, bits, hq, hkv, d, page, dtype):
    q, kv = (STEPS + CHUNKS)[i]
    check(K.problem("cuda", bits, dtype, hq=hq, hkv=hkv, d=d, page=page, q_len=q, kv_len=kv, seed=i, fused=bool(i & 1), extra_tokens=i % 3))


@pytest.mark.parametrize("kind", ["cap", "distance", "prefix", "cap+distance+prefix"])
@pytest.mark.parametrize("q,kv", [((1, 1, 1), (40, 700, 1)), ((60, 1, 130), (61, 800, 400))])
@pytest.mark.parametrize("bits,dtype,hq,hkv,d", [(8, BF, 8, 2, 128), (4, FP, 12, 4, 64), (4, BF, 4, 4, 128), (8, FP, 8, 1, 64)])
def test_scores_over_packed_rows(bits, kind, q, kv, dtype, hq, hkv, d):
    s = K.problem("cuda", bits, dtype, hq=hq, hkv=hkv, d=d, page=16, q_len=q, kv_len=kv, seed=11, hot=6.0)
    check(s, **scores_of(kind, s, q, kv))


@pytest.mark.parametrize("bits,d", [(8, 64), (8, 128), (4, 64), (4, 128)])
@pytest.mark.parametrize("q,kv", [((1, 1), (100, 40)), ((40,), (100,)), ((150, 2), (333, 70))])
def test_packed_rows_that_are_no_numbers(bits, d, q, kv):
    """Keys and values of a sequence's last row are NaN: its token alone sees them; then a seen value is, in one channel (or block)."""
    s = K.problem("cuda", bits, BF, hq=8, hkv=2, d=d, page=16, q_len=q, kv_len=kv, seed=5)
    clean, clean_lse = attend(s)
    last = kv[0] - 1
    page, row = int(s.table[0, last // 16]), q[0] - 1
    K.set_value(s, "v", page, 0, last % 16, 3)
    K.set_value(s, "v", page, 1, last % 16, 40)
    out, lse = check(s)
    keep = torch.arange(s.n, device="cuda") != row
    assert torch.equal(out[keep], clean[keep]) and torch.equal(lse, clean_lse)
    s.k_scale[page, :, last % 16] = 255
    out, lse = attend(s)
    assert torch.equal(out[keep], clean[keep]) and torch.equal(lse[keep], clean_lse[keep])
    assert torch.isnan(out[row]).all() and torch.isnan(lse[row]).all()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q", [1, 5, 150])
def test_absent_packed_pages(q, bits):
    s = K.problem("cuda", bits, BF, hq=8, hkv=2, d=64, page=16, q_len=(q, min(q, 20)), kv_len=(700, 90), seed=4)
    s.table[0, 0], s.table[0, 5], s.table[0, 6], s.table[1, 2] = -1, s.n_pages, 2 ** 31 - 1, -2 ** 31
    check(s)
    s.table[1, :] = -1
    out, lse = check(s)
    assert (lse[q:] == -math.inf).all() and (out[q:] == 0).all()


@pytest.mark.parametrize("bits,hq,hkv,d,q,kv", [(8, 8, 1, 128, (1, 1), (40001, 9)), (4, 16, 2, 64, (1, 3), (30000, 17000)), (8, 4, 2, 128, (40,), (20001,)),
                                               (4, 8, 8, 128, (1,) * 3, (9000, 1, 8191)),
                                               (4, 8, 8, 64, (1,) * 8, (17000, 1, 90, 0, 4097, 300, 2, 8192))])
def test_pieces_of_packed_rows_are_joined(bits, hq, hkv, d, q, kv):
    s = K.problem("cuda", bits, BF, hq=hq, hkv=hkv, d=d, page=64, q_len=q, kv_len=kv, seed=9)
    out, lse = check(s)
    again = attend(s)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


# ---- windows ----------------------------------------------------------------------------------------

WINDOWS = [(1, 0), (1, 1), (5, 4), (16, 0), (33, 17), (128, 4), (130, 64), (1000, 4), (5000, 5000)]


@pytest.mark.parametrize("window,sink", WINDOWS)
@pytest.mark.parametrize("bits,dtype,hq,hkv,d,page", [(16, BF, 8, 2, 128, 16), (16, FP, 12, 4, 64, 32), (8, BF, 8, 1, 128, 64), (4, FP, 3, 3, 64, 16)])
@pytest.mark.parametrize("q,kv", [((1, 1, 1, 0), (1, 700, 2049, 5)), ((2, 33, 7), (2, 300, 1500)), ((300, 1, 129), (2100, 640, 129))])
def test_windows(q, kv, window, sink, bits, dtype, hq, hkv, d, page):
    make = dict(hq=hq, hkv=hkv, d=d, page=page, q_len=q, kv_len=kv, seed=window + sink)
    s = R.problem("cuda", dtype, **make) if bits == 16 else K.problem("cuda", bits, dtype, **make)
    check(s, window, sink)


@pytest.mark.parametrize("kind", ["cap", "distance", "prefix", "cap+distance+prefix"])
@pytest.mark.parametrize("q,kv", [((1, 1, 1), (40, 700, 1)), ((60, 1, 130), (61, 800, 400))])
@pytest.mark.parametrize("bits,dtype,hq,hkv,d", [(16, BF, 8, 2, 128), (16, FP, 12, 4, 64), (4, BF, 4, 4, 128), (8, FP, 8, 1, 64)])
def test_scores_under_a_window(bits, kind, q, kv, dtype, hq, hkv, d):
    make = dict(hq=hq, hkv=hkv, d=d, page=16, q_len=q, kv_len=kv, seed=12, hot=6.0)
    s = R.problem("cuda", dtype, **make) if bits == 16 else K.problem("cuda", bits, dtype, **make)
    check(s, 50, 3, **scores_of(kind, s, q, kv))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("q,kv", [((4,), (1,)), ((1, 3, 40), (0, 1, 7)), ((100, 2), (30, 0)), ((200, 1), (90, 600))])
def test_rows_without_a_slot_see_nothing_under_a_window(q, kv, dtype):
    s = R.problem("cuda", dtype, 8, 2, 64, 16, q, kv, seed=3)
    out, lse = check(s, 9, 2)
    lost = max(0, q[0] - kv[0])
    assert (out[:lost] == 0).all() and (lse[:lost] == -math.inf).all()
    check(s, 9, 2, prefix=torch.tensor([1] * len(q), dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("q,kv", [((1, 1), (3000, 500)), ((90, 2), (2000, 800))])
def test_what_a_window_hides_has_no_influence(q, kv, bits):
    """Neither rows nor table entries: what no token sees is absent, or no number."""
    make = dict(hq=8, hkv=2, d=128, page=16, q_len=q, kv_len=kv, seed=6)
    s = R.problem("cuda", BF, **make) if bits == 16 else K.problem("cuda", bits, BF, **make)
    window, sink = 100, 20
    out, lse = check(s, window, sink)
    for b, (a, t) in enumerate(zip(q, kv)):
        first = (t - a - window + 1) // 16             # the page that the first token's window begins in
        s.table[b, 2:first] = torch.tensor([-1, s.n_pages, 2 ** 30] * 100, dtype=torch.int32)[:max(0, first - 2)].cuda()
        for j in list(range(sink, 32)) + list(range(16 * first, t - a - window + 1)):
            page = int(s.table[b, j // 16])
            if bits == 16:
                s.k[page, :, j % 16], s.v[page, :, j % 16] = math.nan, math.inf
            else:
                s.k_scale[page, :, j % 16], s.v_scale[page, :, j % 16] = 255, 255
    again = attend(s, window, sink)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("q,kv", [((1, 1), (900, 31)), ((70, 3), (700, 64))])
@pytest.mark.parametrize("bits", [16, 4])
def test_a_window_that_reaches_the_first_row_is_none(bits, q, kv):
    make = dict(hq=8, hkv=2, d=64, page=16, q_len=q, kv_len=kv, seed=7)
    s = R.problem("cuda", BF, **make) if bits == 16 else K.problem("cuda", bits, BF, **make)
    ref, rl, tol, ltol = K.attention(s)
    for window, sink in [(0, 0), (0, 5), (max(kv), 0), (2 ** 31 - 1, 2 ** 31 - 1)]:
        out, lse = attend(s, window, sink)
        R.close(out, ref, tol, "out")
        R.close(lse, rl, ltol, "lse")


# ---- trees ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("window,sink", [(0, 0), (40, 4)])
@pytest.mark.parametrize("bits,dtype,hq,hkv,d,page", [(16, BF, 8, 2, 128, 16), (16, FP, 12, 4, 64, 32), (8, BF, 8, 1, 128, 64), (4, FP, 3, 3, 64, 16)])
@pytest.mark.parametrize("q,kv", [((2,), (2,)), ((3, 1, 0, 4), (300, 90, 0, 4)), ((25,), (1000,)), ((64, 65, 1), (64, 700, 33)), ((200, 5), (431, 2049))])
def test_trees(q, kv, bits, dtype, hq, hkv, d, page, window, sink):
    make = dict(hq=hq, hkv=hkv, d=d, page=page, q_len=q, kv_len=kv, seed=sum(q), extra_tokens=1)
    s = R.problem("cuda", dtype, **make) if bits == 16 else K.problem("cuda", bits, dtype, **make)
    check(s, window, sink, K.drafts(s, seed=1))


@pytest.mark.parametrize("q,kv", [((3, 2), (40, 3)), ((40, 70), (40, 300))])
def test_any_bits_are_a_tree(q, kv):
    """Bits of tokens behind, of none, of itself alone, and bits behind the sequence's tokens."""
    s = R.problem("cuda", BF, 8, 2, 64, 16, q, kv, seed=2)
    g = torch.Generator().manual_seed(3)
    tree = torch.rand(s.n, 128, generator=g) < 0.3
    tree[0] = False                                    # with no context before it, this row sees nothing
    tree[1] = True
    out, lse = check(s, 0, 0, tree)
    if kv[0] == q[0]:
        assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    check(s, 7, 2, tree)
    check(s, 0, 0, tree, **scores_of("cap+distance+prefix", s, q, kv))


def test_trees_whose_first_tokens_have_no_slot():
    s = R.problem("cuda", FP, 8, 2, 64, 16, (9, 70), (4, 30), seed=2)
    tree = torch.rand(s.n, 70, generator=torch.Generator().manual_seed(4)) < 0.5
    out, lse = check(s, 0, 0, tree)
    assert (out[:5] == 0).all() and (out[9:49] == 0).all()
    check(s, 3, 1, tree)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("q,kv", [((3,), (100,)), ((40, 7), (300, 90))])
def test_a_chain_of_drafts_is_causal(q, kv, bits):
    make = dict(hq=8, hkv=2, d=128, page=16, q_len=q, kv_len=kv, seed=2)
    s = R.problem("cuda", BF, **make) if bits == 16 else K.problem("cuda", bits, BF, **make)
    tree = torch.zeros(s.n, s.max_q, dtype=torch.bool)
    for b, a in enumerate(q):
        for i in range(a):
            tree[sum(q[:b]) + i, :i + 1] = True
    ref, rl, tol, ltol = K.attention(s)
    out, lse = attend(s, tree=tree)
    R.close(out, ref, tol, "out")
    R.close(lse, rl, ltol, "lse")


@pytest.mark.parametrize("q,kv", [((25,), (300,)), ((4, 3), (100, 50))])
def test_hidden_drafts_have_no_influence(q, kv):
    """A draft that is no number: those that do not descend from it are as they were, to the bit."""
    s = R.problem("cuda", BF, 8, 2, 64, 16, q, kv, seed=5)
    tree = K.drafts(s, seed=3)
    clean = attend(s, tree=tree)
    slot = kv[0] - q[0] + 1                            # the first sequence's second draft
    page = int(s.table[0, slot // 16])
    s.k[page, :, slot % 16] = math.nan
    s.v[page, :, slot % 16] = math.inf
    out, lse = attend(s, tree=tree)
    sees = tree[:, 1].clone()
    sees[q[0]:] = False
    sees = sees.cuda()
    assert sees.any() and torch.equal(out[~sees], clean[0][~sees]) and torch.equal(lse[~sees], clean[1][~sees])
    assert torch.isnan(out[sees]).all()


# ---- batches, streams, graphs -----------------------------------------------------------------------

@pytest.mark.parametrize("bits,hq,hkv,d", [(8, 8, 2, 128), (4, 4, 1, 64), (16, 8, 8, 64)])
def test_batches_of_more_than_64_sequences(bits, hq, hkv, d):
    q = [1 if b % 7 else 30 + b % 5 for b in range(150)]
    q[40] = q[149] = 0
    kv = [max(a, 37 * b % 200) for b, a in enumerate(q)]
    make = dict(hq=hq, hkv=hkv, d=d, page=16, q_len=q, kv_len=kv, seed=5)
    s = R.problem("cuda", BF, **make) if bits == 16 else K.problem("cuda", bits, BF, **make)
    check(s, 30, 2)
    if bits != 16:
        check(s)
        pages, batch, _ = handles(s)
        k, v = (torch.empty(s.n, hkv, d, dtype=BF, device="cuda") for _ in "kv")
        P.arkv_packed_read(pages, batch, k, v)
        for b, a in enumerate(q):
            for h in range(hkv if a else 0):
                assert torch.equal(k[sum(q[:b]):sum(q[:b]) + a, h], R.rows(s, s.k, b, h)[0][kv[b] - a:])
                assert torch.equal(v[sum(q[:b]):sum(q[:b]) + a, h], R.rows(s, s.v, b, h)[0][kv[b] - a:])


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("q,kv", [((1, 1, 1), (700, 3, 90)), ((5, 0, 2), (300, 8, 2)), ((40, 3), (900, 40)), ((150, 1), (2000, 1500))])
def test_bounds_may_be_loose(q, kv, bits):
    """What is announced shapes the launches, not the results: tokens and rows of sequences far below their bounds."""
    make = dict(hq=16, hkv=2, d=128, page=32, q_len=q, kv_len=kv, seed=4, width=200)
    s = R.problem("cuda", BF, **make) if bits == 16 else K.problem("cuda", bits, BF, **make)
    tree = K.drafts(s)
    for window, drafted, max_kv in [(0, True, 6400), (50, False, 6400), (50, True, 4000), (0, True, max(kv))]:
        ref, rl, tol, ltol = K.attention(s, window, 4, tree if drafted else None)
        pages, batch, ws = handles(s, max_q=s.n, max_kv=max_kv)
        out, lse = torch.empty(s.n, s.hq, s.d, dtype=BF, device="cuda"), torch.empty(s.n, s.hq, device="cuda")
        wide = torch.zeros(s.n, -(-s.n // 64) * 64, dtype=torch.bool)
        wide[:, :tree.shape[1]] = tree
        sight = P.arkv_sight(window, 4, K.words(wide).cuda() if drafted else None)
        if bits == 16:
            P.arkv_paged_attention_sight(pages, batch, sight, s.q, s.scale, out, lse=lse, workspace=ws)
        else:
            P.arkv_packed_attention(pages, batch, s.q, s.scale, out, lse=lse, sight=sight, workspace=ws)
        R.close(out, ref, tol, "out")
        R.close(lse, rl, ltol, "lse")


def test_one_workspace_serves_every_batch_bits_and_sight():
    s0 = K.problem("cuda", 8, BF, hq=16, hkv=4, d=128, page=16, q_len=(300,) * 6, kv_len=(3000,) * 6, seed=1)
    ws = handles(s0)[2]
    for i, (bits, q, kv, window, drafted) in enumerate([(8, (1,), (2900,), 0, 0), (4, (250, 1), (3000, 1), 0, 0), (16, (40,), (2000,), 300, 0), (8, (64, 20), (900, 2999), 0, 1),
                                                        (4, (1,) * 6, (3000,) * 6, 64, 0), (16, (8,), (3000,), 0, 1)]):
        make = dict(hq=16, hkv=4, d=128, page=16, q_len=q, kv_len=kv, seed=i)
        s = R.problem("cuda", BF, **make) if bits == 16 else K.problem("cuda", bits, BF, **make)
        tree = K.drafts(s) if drafted else None
        out, lse = attend(s, window, 4 if window else 0, tree, ws=ws)
        ref, rl, tol, ltol = K.attention(s, window, 4, tree)
        R.close(out, ref, tol, "out")
        R.close(lse, rl, ltol, "lse")


def test_another_stream_repeats_to_the_bit():
    s = K.problem("cuda", 4, BF, hq=16, hkv=2, d=128, page=16, q_len=(40, 1, 1), kv_len=(900, 5000, 20), seed=3)
    tree = K.drafts(s)
    first = attend(s, 200, 4, tree)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        second = attend(s, 200, 4, tree)
    torch.cuda.synchronize()
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])


@pytest.mark.parametrize("bits", [8, 4])
def test_a_captured_step_follows_lengths_tables_and_drafts(bits):
    """append, attention of drafts under a window, reading back, in one graph, replayed with other lengths, pages, rows and trees."""
    hq, hkv, d, page, B, most = 8, 2, 64, 16, 3, 12
    pages = pool(bits, 40, hkv, page, d, BF, fill=0)
    table = torch.full((B, 10), -1, dtype=torch.int32, device="cuda")
    cu, kv_len = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    n = B * most
    qkv = torch.zeros(n, hq + 2 * hkv, d, dtype=BF, device="cuda")
    positions, bits_of = torch.zeros(1, n, dtype=torch.int32, device="cuda"), torch.zeros(n, 1, dtype=torch.int64, device="cuda")
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).cuda()
    rotary, sight = P.arkv_rotary(freq), P.arkv_sight(60, 4, bits_of)
    batch = P.arkv_page_batch(cu, kv_len, table, n, most, 160)
    ws = P.arkv_packed_workspace(pages, batch, hq)
    q, out, k, v = (torch.zeros(n, h, d, dtype=BF, device="cuda") for h in (hq, hq, hkv, hkv))
    lse = torch.zeros(n, hq, device="cuda")

    def step():
        P.arkv_packed_append(pages, batch, rotary, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], positions, q)
        P.arkv_packed_attention(pages, batch, q, 0.125, out, lse=lse, sight=sight, workspace=ws)
        P.arkv_packed_read(pages, batch, k, v)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(0)
    have = [0] * B
    for turn in range(4):
        q_len = [int(torch.randint(0, most + 1, (1,), generator=g)) for _ in range(B)]
        have = [a + b for a, b in zip(have, q_len)]
        order = torch.randperm(40, generator=g)[:30].reshape(3, 10).to(torch.int32) if turn == 0 else table.cpu()
        table.copy_(order)
        cu.copy_(torch.tensor([sum(q_len[:b]) for b in range(B + 1)], dtype=torch.int32))
        kv_len.copy_(torch.tensor(have, dtype=torch.int32))
        qkv.copy_(torch.randn(n, hq + 2 * hkv, d, generator=g).to(BF))
        positions.copy_(torch.randint(0, 1000, (1, n), generator=g, dtype=torch.int32))
        bits_of.copy_(torch.randint(0, 1 << most, (n, 1), generator=g))
        results = []
        for run in (graph.replay, step):
            for x in (out, k, v, q):
                x.fill_(3.0)
            lse.fill_(3.0)
            run()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (out, lse, k, v, q, pages.k, pages.v, pages.k_scale, pages.v_scale, pages.pos)])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        assert not (results[0][0][:sum(q_len)] == 3).all() or not sum(q_len)


def test_a_batch_without_new_tokens():
    s = K.problem("cuda", 8, BF, hq=4, hkv=2, d=64, page=16, q_len=(0, 0), kv_len=(30, 0), seed=1)
    pages, batch, ws = handles(s)
    z = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    q = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    P.arkv_packed_append(pages, batch, P.arkv_rotary(None), q, z, z, torch.empty(1, 0, dtype=torch.int32, device="cuda"), q)
    P.arkv_packed_read(pages, batch, z, z)
    P.arkv_packed_attention(pages, batch, q, 0.125, torch.empty_like(q), sight=P.arkv_sight(5, 1, torch.empty(0, 1, dtype=torch.int64, device="cuda")), workspace=ws)
    torch.cuda.synchronize()


def test_arguments_on_the_gpu_are_checked():
    s = K.problem("cuda", 8, BF, hq=4, hkv=2, d=64, page=16, q_len=(3,), kv_len=(30,), seed=1)
    pages, batch, ws = handles(s)
    out = torch.empty(3, 4, 64, dtype=BF, device="cuda")
    for kw in [dict(sight=P.arkv_sight(tree=torch.zeros(2, 1, dtype=torch.int64, device="cuda"))), dict(lse=torch.empty(3, 2, device="cuda")),
               dict(slopes=torch.ones(4, device="cuda"))]:
        with pytest.raises(ValueError):
            P.arkv_packed_attention(pages, batch, s.q, 0.1, out, workspace=ws, **kw)
    with pytest.raises(ValueError):
        P.arkv_packed_attention(pages, batch, s.q.to(FP), 0.1, out, workspace=ws)
    with pytest.raises(P.ArkvError):
        P.arkv_packed_attention(pages, batch, s.q, 0.1, out, workspace=ws[:TICKETS - 16])
    with pytest.raises(P.ArkvError):
        P.arkv_packed_attention(pages, batch, s.q, 0.1, out, sight=P.arkv_sight(-1), workspace=ws)
    with pytest.raises(ValueError):
        P.arkv_packed_read(pages, batch, out, None)
    with pytest.raises(ValueError):
        P.arkv_packed_pages(s.k_codes, s.v_codes, s.k_scale[..., :1].contiguous(), s.v_scale, s.pos, BF)


# ---- a run of them together ---------------------------------------------------------------------------

@pytest.mark.parametrize("bits,dtype", [(8, BF), (4, BF), (8, FP)])
def test_rounds_of_drafts_leave_what_their_accepted_tokens_would(bits, dtype):
    """Drafting, attending and accepting, against a twin that never drafted: the same rows, to the bit, and the same outputs."""
    from paper_2603_08727_amd.paged_drafts_example import DraftedLayer
    make = lambda: DraftedLayer(3, hidden=128, bits=bits, rows=192, window=40, sink=4, max_tokens=70, dtype=dtype, seed=3)  # noqa: E731
    layer, twin = make(), make()
    g = torch.Generator().manual_seed(1)
    new = lambda n: torch.randn(n, 128, generator=g).to(dtype).cuda()  # noqa: E731
    x = new(50 + 3 + 70)
    assert torch.equal(layer.prompt(x, [50, 3, 70]), twin.prompt(x, [50, 3, 70]))
    chosen = [[[-1, 0, 0, 1, 2, 4], [0, 2, 4]], [[-1, 0], []], [[-1, -1, 1, 2], [1, 2]]]
    for turn in range(3):
        parents, paths = [c[0] for c in chosen], [c[1] for c in chosen]
        q_len = [len(p) for p in parents]
        x = new(sum(q_len))
        y = layer.draft(x, parents)
        layer.accept(paths)
        picked = [sum(q_len[:r]) + i for r, path in enumerate(paths) for i in path]
        z = twin.prompt(x[picked], [len(p) for p in paths])
        # An accepted draft saw what the accepted token sees.  On either side an output is off by its rounding and by those of the probabilities, 2 U
        # of the largest value, and 2^-12 of it covers sums and logits in 32 bits; the projection rounds once more.
        most = float(max(K.values(c.cpu(), s.cpu(), bits).abs().max() for c, s in ((twin.pages.v, twin.pages.v_scale),)))
        off = 2 * (2 * R.U[dtype] + 2.0 ** -12) * most * math.sqrt(len(picked) * twin.hq * twin.d)
        w = float(torch.linalg.matrix_norm(twin.w_out.float(), 2))
        assert (y[picked].float() - z.float()).norm() <= w * off + 3 * R.U[dtype] * z.float().norm()
        assert layer.have == twin.have
        kv = torch.tensor(layer.have, dtype=torch.int32, device="cuda")
        cu = torch.tensor([sum(layer.have[:r]) for r in range(4)], dtype=torch.int32, device="cuda")
        n = sum(layer.have)
        rows = []
        for each in (layer, twin):
            k, v = (torch.empty(n, each.hkv, each.d, dtype=dtype, device="cuda") for _ in "kv")
            P.arkv_packed_read(each.pages, P.arkv_page_batch(cu, kv, each.table, n, max(layer.have), max(layer.have)), k, v)
            rows.append((k, v))
        assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
    x = new(3)
    assert torch.equal(layer.prompt(x, [1, 1, 1]), twin.prompt(x, [1, 1, 1]))
    with pytest.raises(ValueError, match="follows"):
        layer.draft(new(2), [[0], [-1], []])


def test_the_drafts_example_runs(capsys):
    from paper_2603_08727_amd import paged_drafts_example
    paged_drafts_example.main()
    assert "round 7" in capsys.readouterr().out
