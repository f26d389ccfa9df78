"""GPU tests of the operators around a paged cache against plain 64-bit forms (tests/paged_ref.py)."""
import math

import pytest
import torch

from paper_2603_08727_amd import paged as P
import paged_ref as R

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
TICKETS = 1 << 16                                      # bytes of a workspace that are zero between calls


def handles(s, max_q=None, max_kv=None):
    pages = P.arkv_pages(s.k, s.v, s.pos, s.weight)
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, s.max_q if max_q is None else max_q, s.max_kv if max_kv is None else max_kv)
    return pages, batch, P.arkv_paged_workspace(pages, batch, s.hq)


def attend(s, **kw):
    pages, batch, ws = handles(s)
    ws[TICKETS:].fill_(0xFF)                           # what a workspace holds behind its tickets does not matter
    out = torch.full((s.n, s.hq, s.d), 7.0, dtype=s.dtype, device="cuda")
    lse = torch.full((s.n, s.hq), 7.0, device="cuda")
    P.arkv_paged_attention(pages, batch, s.q, s.scale, out, lse=lse, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert not ws[:TICKETS].any()
    return out, lse


def check_attention(s, **kw):
    out, lse = attend(s, **kw)
    ref, rl, tol, ltol = R.attention(s, **kw)
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


STEPS = [((1,), (1,)), ((1,), (2,)), ((1,), (15,)), ((1,), (16,)), ((1,), (17,)), ((1, 1, 1), (63, 64, 65)), ((1, 1), (1000, 31)),
         ((1, 0, 1, 1), (129, 0, 513, 2)), ((1,) * 9, (5, 700, 33, 1, 2049, 64, 96, 128, 300))]
CHUNKS = [((2,), (2,)), ((3,), (50,)), ((16, 1), (16, 40)), ((17,), (17,)), ((33, 0, 5), (64, 0, 5)), ((64,), (1000,)), ((129, 1, 77), (300, 1025, 77)),
          ((300,), (2100,)), ((5, 1, 1, 40), (900, 3, 700, 41)), ((257,), (257,))]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 64, 16), (8, 2, 128, 32), (3, 3, 128, 16), (12, 4, 64, 64), (16, 1, 64, 128), (10, 2, 128, 16),
                                           (16, 2, 128, 256)])
@pytest.mark.parametrize("i", range(len(STEPS)))
def test_steps_of_single_tokens(i, hq, hkv, d, page, dtype):
    q, kv = STEPS[i]
    check_attention(R.problem("cuda", dtype, hq, hkv, d, page, q, kv, seed=i, fused=bool(i & 1)))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 64, 16), (4, 1, 128, 32), (3, 3, 128, 16), (12, 4, 64, 64), (16, 1, 64, 1024), (7, 1, 128, 16)])
@pytest.mark.parametrize("i", range(len(CHUNKS)))
def test_chunks(i, hq, hkv, d, page, dtype):
    q, kv = CHUNKS[i]
    check_attention(R.problem("cuda", dtype, hq, hkv, d, page, q, kv, seed=i, fused=bool(i & 1), extra_tokens=i % 3))


@pytest.mark.parametrize("kind", ["cap", "distance", "prefix", "cap+distance", "cap+prefix", "distance+prefix", "all"])
@pytest.mark.parametrize("i,q,kv", [(0, (1, 1, 1), (40, 700, 1)), (1, (60, 1, 130), (61, 800, 400)), (2, (200,), (1500,))])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 8, 2, 128), (FP, 12, 4, 64), (FP, 4, 4, 128), (BF, 8, 1, 64)])
def test_scores(kind, i, q, kv, dtype, hq, hkv, d):
    s = R.problem("cuda", dtype, hq, hkv, d, 16, q, kv, seed=10 + i, hot=6.0)
    kw = {}
    if "cap" in kind or kind == "all":
        kw["cap"] = 3.5
    if "distance" in kind or kind == "all":
        kw["slopes"], kw["q_pos"] = slopes_of(s)
    if "prefix" in kind or kind == "all":
        pre = [min(t, t - a + (2 * a) // 3) for a, t in zip(q, kv)]
        pre[0] = kv[0] + 9                              # longer than what is cached: cut
        if len(pre) > 1:
            pre[1] = -4 if i else 3                     # nothing beyond the causal ones
        kw["prefix"] = torch.tensor(pre, dtype=torch.int32, device="cuda")
    check_attention(s, **kw)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("q,kv", [((4,), (1,)), ((1, 3, 40), (0, 1, 7)), ((100, 2), (30, 0)), ((200, 1), (90, 600))])
def test_rows_that_see_nothing(q, kv, dtype):
    """More new tokens than slots: the first have none and see nothing (or the prefix alone)."""
    s = R.problem("cuda", dtype, 8, 2, 64, 16, q, kv, seed=3)
    out, lse = check_attention(s)
    lost = max(0, q[0] - kv[0])
    assert (out[:lost] == 0).all() and (lse[:lost] == -math.inf).all()
    s = R.problem("cuda", dtype, 8, 2, 64, 16, q, kv, seed=3)
    check_attention(s, prefix=torch.tensor([1] * len(q), dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype,d", [(BF, 64), (FP, 128), (BF, 128)])
@pytest.mark.parametrize("q", [1, 5, 150])
def test_absent_pages(q, dtype, d):
    s = R.problem("cuda", dtype, 8, 2, d, 16, (q, min(q, 20)), (700, 90), seed=4)
    s.table[0, 0], s.table[0, 5], s.table[0, 6], s.table[1, 2] = -1, s.n_pages, 2 ** 31 - 1, -2 ** 31
    check_attention(s)
    s.table[1, :] = -1                                 # a sequence whose pages are all gone
    out, lse = check_attention(s)
    assert (lse[q:] == -math.inf).all() and (out[q:] == 0).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("q,kv", [((40,), (100,)), ((150,), (333,)), ((2,), (70,))])
def test_unseen_rows_have_no_influence(q, kv, what, dtype):
    """Keys and values of the last new token are no numbers: only its own row, which sees them, may show it."""
    s = R.problem("cuda", dtype, 8, 2, 64, 16, q, kv, seed=5)
    clean, clean_lse = attend(s)
    last = kv[0] - 1
    page = int(s.table[0, last // 16])
    s.v[page, :, last % 16, 3] = what
    s.v[page, 0, last % 16, 40] = what
    out, lse = check_attention(s)
    assert torch.equal(out[:-1], clean[:-1]) and torch.equal(lse, clean_lse)
    s.k[page, :, last % 16] = math.nan
    out, lse = attend(s)
    assert torch.equal(out[:-1], clean[:-1]) and torch.equal(lse[:-1], clean_lse[:-1])
    assert torch.isnan(out[-1]).all() and torch.isnan(lse[-1]).all()


@pytest.mark.parametrize("q,kv", [((1,), (5000,)), ((70,), (3000,))])
def test_values_that_are_seen_but_no_numbers_reach_their_channel_alone(q, kv):
    s = R.problem("cuda", BF, 8, 2, 128, 16, q, kv, seed=6)
    page = int(s.table[0, 10])
    s.v[page, 1, 3, 77] = math.inf
    out, _ = attend(s)
    bad = ~torch.isfinite(out.float())
    want = torch.zeros_like(bad)
    want[:, 4:, 77] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("q", [1, 90])
def test_extreme_logits(q):
    """Rows whose logits reach thousands, and rows of equal logits."""
    s = R.problem("cuda", BF, 8, 2, 128, 16, (q, q), (900, 333), seed=7, hot=300.0)
    check_attention(s)
    s.q.zero_()
    check_attention(s)
    s = R.problem("cuda", BF, 8, 2, 128, 16, (q,), (900,), seed=8, hot=200.0)
    s.scale = -s.scale
    check_attention(s)


@pytest.mark.parametrize("q,kv,hq,hkv", [((1, 1), (20001, 70001), 8, 1), ((500,), (9000,), 8, 2), ((1, 600, 1), (40000, 4001, 7), 4, 2)])
def test_long_caches(q, kv, hq, hkv):
    check_attention(R.problem("cuda", BF, hq, hkv, 128, 64, q, kv, seed=9))
    s = R.problem("cuda", FP, hq, hkv, 64, 64, q, kv, seed=9)
    sl, qp = slopes_of(s)
    check_attention(s, slopes=sl, q_pos=qp)


@pytest.mark.parametrize("lens", [(1025,), (2048,), (4100,), (2049, 1, 5000, 0, 1024), (1500,) * 40, (30000,), (33000, 70)])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 8, 2, 128), (FP, 16, 1, 64)])
def test_pieces_are_joined(lens, dtype, hq, hkv, d):
    """Sequences of one piece, of a few (joined by the last workgroup) and of many (by a launch), the same workspace again and again."""
    s = R.problem("cuda", dtype, hq, hkv, d, 16, tuple(min(1, t) for t in lens), lens, seed=13)
    out, lse = check_attention(s)
    pages, batch, ws = handles(s)
    for _ in range(5):
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        P.arkv_paged_attention(pages, batch, s.q, s.scale, o2, lse=l2, workspace=ws)
        assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("q,kv", [((17,), (600,)), ((128,), (1025,)), ((200, 1, 0, 130), (2000, 3000, 0, 257)), ((300,) * 3, (300, 2600, 900)),
                                  ((20,), (9001,)), ((33, 1), (70001, 40000)), ((1, 1, 19), (5000, 16, 4500))])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 8, 2, 128), (FP, 12, 4, 64), (BF, 1, 1, 128)])
def test_pieces_of_chunks_are_joined(q, kv, dtype, hq, hkv, d):
    """Blocks of rows whose keys are a few workgroups' (the last one joins them) or many; the same workspace again and again."""
    s = R.problem("cuda", dtype, hq, hkv, d, 16, q, kv, seed=16)
    out, lse = check_attention(s)
    pages, batch, ws = handles(s)
    for i in range(4):
        ws[TICKETS:].fill_(0xFF)
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        P.arkv_paged_attention(pages, batch, s.q, s.scale, o2, lse=l2, workspace=ws)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        assert not ws[:TICKETS].any()


def test_one_workspace_for_batches_of_any_shape():
    big = R.problem("cuda", BF, 8, 8, 128, 16, (1,) * 20, (3000,) * 20, seed=14)
    small = R.problem("cuda", BF, 8, 2, 128, 16, (100, 1), (5000, 2100), seed=15)
    want = [attend(big), attend(small)]
    ws = torch.zeros(max(handles(s)[2].numel() for s in (big, small)), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        for s, (out, lse) in zip((big, small), want):
            pages, batch, _ = handles(s)
            o2, l2 = torch.empty_like(out), torch.empty_like(lse)
            P.arkv_paged_attention(pages, batch, s.q, s.scale, o2, lse=l2, workspace=ws)
            assert torch.equal(out, o2) and torch.equal(lse, l2)
            P.arkv_paged_weights(pages, batch, s.q, s.scale, l2, workspace=ws)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB, its last pages in use."""
    n_pages, hkv, page, d = 40000, 8, 64, 128
    small = R.problem("cuda", BF, 16, hkv, d, page, (3, 1), (200, 130), seed=11)
    k = torch.empty((n_pages, hkv, page, d), dtype=BF, device="cuda")
    v = torch.empty_like(k)
    base = n_pages - small.n_pages
    k[base:], v[base:] = small.k, small.v
    out, lse = attend(small)
    pos = torch.zeros((n_pages, hkv, page), dtype=torch.int32, device="cuda")
    weight = torch.zeros((n_pages, hkv, page), device="cuda")
    pos[base:], weight[base:] = small.pos, small.weight
    big = R.problem("cuda", BF, 16, hkv, d, page, (3, 1), (200, 130), seed=11)
    big.k, big.v, big.pos, big.weight, big.n_pages = k, v, pos, weight, n_pages
    big.table = torch.where(small.table >= 0, small.table + base, small.table)
    o2, l2 = attend(big)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    for s in (small, big):
        pages, batch, ws = handles(s)
        P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.5, workspace=ws)
        new = torch.randn(s.n, hkv, d, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
        P.arkv_paged_append(pages, batch, P.arkv_rotary(None), None, new, new, torch.arange(s.n, dtype=torch.int32, device="cuda")[None], None)
    assert torch.equal(big.weight[base:].nan_to_num(9.0), small.weight.nan_to_num(9.0))
    assert torch.equal(big.k[base:].float().nan_to_num(9.0), small.k.float().nan_to_num(9.0))
    dst = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    kept, lens = torch.empty((2, hkv, 100), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    P.arkv_paged_evict(P.arkv_pages(big.k, big.v, big.pos, big.weight), handles(big)[1], torch.tensor([100, 100], dtype=torch.int32, device="cuda"),
                       dst, kept, lens)
    ref, _ = R.evict(big, [100, 100], 4, 32, 100)
    assert torch.equal(kept.cpu(), ref)
    old = R.rows(big, big.k, 0, 7)[0]
    assert torch.equal(big.k[0, 7], old[kept[0, 7, :64].long()])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 64, 16), (8, 2, 128, 64), (3, 3, 128, 16), (12, 4, 64, 32), (16, 1, 128, 16)])
@pytest.mark.parametrize("i", range(6))
def test_weights(i, hq, hkv, d, page, dtype):
    q, kv = [((1,), (1,)), ((1, 1, 0, 1), (64, 700, 0, 33)), ((33, 1, 90), (400, 1025, 90)), ((300,), (2100,)), ((40, 3), (7, 0)), ((130,), (130,))][i]
    s = R.problem("cuda", dtype, hq, hkv, d, page, q, kv, seed=20 + i, fused=bool(i & 1), extra_tokens=i % 2)
    _, lse = attend(s)
    pages, batch, ws = handles(s)
    ws[TICKETS:].fill_(0xFF)
    for decay, other in [(1.0, False), (0.0, False), (0.75, True)]:
        carried = torch.rand_like(s.weight) if other else s.weight.clone()
        ref, tol = R.weights(s, lse, decay, carried)
        P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=decay, carried=carried if other else None, workspace=ws)
        R.close(s.weight, ref, tol, "weight")


@pytest.mark.parametrize("kind", ["cap", "distance", "prefix", "all"])
@pytest.mark.parametrize("q,kv", [((1, 1), (40, 700)), ((60, 1, 130), (61, 800, 400))])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 8, 2, 128), (FP, 12, 4, 64), (BF, 8, 1, 64)])
def test_weights_of_scores(kind, q, kv, dtype, hq, hkv, d):
    s = R.problem("cuda", dtype, hq, hkv, d, 16, q, kv, seed=30, hot=4.0)
    kw = {}
    if kind in ("cap", "all"):
        kw["cap"] = 3.5
    if kind in ("distance", "all"):
        kw["slopes"], kw["q_pos"] = slopes_of(s)
    if kind in ("prefix", "all"):
        kw["prefix"] = torch.tensor([min(t, t - a + (2 * a) // 3) for a, t in zip(q, kv)], dtype=torch.int32, device="cuda")
    _, lse = attend(s, **kw)
    pages, batch, ws = handles(s)
    ref, tol = R.weights(s, lse, 1.0, s.weight, **kw)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, workspace=ws, **kw)
    R.close(s.weight, ref, tol, "weight")


@pytest.mark.parametrize("lens", [(0, 0), (1, 0), (3, 40), (0, 64)])
def test_sequences_shorter_than_announced(lens):
    """Bounds that say 64 new tokens each for all sequences, lengths that say less: nobody is left out."""
    s = R.problem("cuda", BF, 8, 2, 64, 16, lens, (300, 90), seed=33, extra_tokens=128 - sum(lens))
    s.max_q = 64
    _, lse = check_attention(s)
    pages, batch, ws = handles(s)
    ref, tol = R.weights(s, lse, 0.5, s.weight)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.5, workspace=ws)
    R.close(s.weight, ref, tol, "weight")


def test_a_batch_without_new_tokens():
    s = R.problem("cuda", BF, 8, 2, 64, 16, (0, 0), (40, 0), seed=34)
    pages, batch, ws = handles(s)
    before = {n: getattr(s, n).clone() for n in ("k", "v", "pos")}
    new, lse = torch.empty(0, 2, 64, dtype=BF, device="cuda"), torch.empty(0, 8, device="cuda")
    P.arkv_paged_append(pages, batch, P.arkv_rotary(None), s.q, new, new, torch.empty(1, 0, dtype=torch.int32, device="cuda"), torch.empty_like(s.q))
    P.arkv_paged_attention(pages, batch, s.q, s.scale, torch.empty_like(s.q), lse=lse, workspace=ws)
    ref, tol = R.weights(s, lse, 0.5, s.weight)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.5, workspace=ws)
    R.close(s.weight, ref, tol, "weight")
    for name, old in before.items():
        assert torch.equal(getattr(s, name).view(torch.uint8), old.view(torch.uint8)), name


def test_weights_of_a_step_sum_to_the_tokens_and_heads():
    s = R.problem("cuda", BF, 8, 2, 128, 16, (50, 1), (333, 1000), seed=31)
    _, lse = attend(s)
    pages, batch, ws = handles(s)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.0, workspace=ws)
    for b, q in enumerate((50, 1)):
        for h in range(2):
            assert abs(float(R.rows(s, s.weight, b, h)[0].double().sum()) - 4 * q) < 1e-3 * q


def test_absent_pages_and_unseen_rows_in_weights():
    s = R.problem("cuda", BF, 8, 2, 64, 16, (5,), (300,), seed=32)
    s.table[0, 3] = -1
    _, lse = attend(s)
    pages, batch, ws = handles(s)
    page = int(s.table[0, 299 // 16])
    s.k[page, :, 299 % 16] = math.nan                  # the last token's key: the rows before it do not see it
    ref, tol = R.weights(s, lse, 1.0, s.weight)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, workspace=ws)
    assert torch.isnan(s.weight[page, :, 299 % 16]).all()
    ref[page, :, 299 % 16] = math.nan
    R.close(s.weight, ref, tol, "weight")


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("axes,rot", [(1, None), (3, None), (2, 32), (4, 48), (1, 0)])
@pytest.mark.parametrize("q,kv", [((1,), (1,)), ((1, 0, 1), (17, 0, 300)), ((33, 5, 100), (40, 5, 250))])
def test_append(q, kv, axes, rot, adjacent, dtype, d):
    s = R.problem("cuda", dtype, 6, 3, d, 16, q, kv, seed=40, extra_tokens=2, fused=True)
    rot = d if rot is None else rot
    half = rot // 2
    g = torch.Generator().manual_seed(1)
    freq = (500000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).cuda()
    axis = [i % axes for i in range(half)]
    positions = torch.randint(0, 200000, (axes, s.n), generator=g, dtype=torch.int32)
    positions[0, 0] = 2 ** 31 - 1
    positions = positions.cuda()
    kv_new = torch.randn(s.n, 9, d, generator=g).to(dtype).cuda()
    kn, vn = kv_new[:, 1:7:2], kv_new[:, 6:]           # strided heads
    pages, batch, _ = handles(s)
    before = {n: getattr(s, n).clone() for n in ("k", "v", "pos", "weight")}
    q_out = torch.full((s.n, 6, d), 7.0, dtype=dtype, device="cuda")
    P.arkv_paged_append(pages, batch, P.arkv_rotary(freq if half else None, axis, axes, adjacent), s.q, kn, vn, positions, q_out)
    n = sum(q)
    (rq, tq), (rk, tk) = (R.rotate(x, positions, freq, axis, adjacent) for x in (s.q, kn))
    R.close(q_out[:n], rq[:n], tq[:n], "q")
    assert (q_out[n:] == 7).all()
    assert torch.equal(q_out[:n, :, rot:], s.q[:n, :, rot:])
    at = 0
    for b, (a, t) in enumerate(zip(q, kv)):
        for i in range(a):
            slot = t - a + i
            page, off = int(s.table[b, slot // 16]), slot % 16
            R.close(s.k[page, :, off], rk[at + i], tk[at + i], "k")
            assert torch.equal(s.v[page, :, off], vn[at + i])
            assert (s.pos[page, :, off] == positions[0, at + i]).all() and (s.weight[page, :, off] == 0).all()
            for name in before:                        # put back: what is left must be untouched
                getattr(s, name)[page, :, off] = before[name][page, :, off]
        at += a
    for name in before:
        assert torch.equal(getattr(s, name).view(torch.uint8), before[name].view(torch.uint8)), name


def test_append_in_place_without_queries_and_without_slots():
    s = R.problem("cuda", BF, 4, 2, 64, 16, (5, 2), (3, 40), seed=41)
    s.table[1, 2] = -1                                 # the second sequence's new tokens have no page
    freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).cuda()
    pos = torch.arange(7, dtype=torch.int32, device="cuda")[None].contiguous()
    kn, vn = torch.randn(7, 2, 64, device="cuda").to(BF), torch.randn(7, 2, 64, device="cuda").to(BF)
    pages, batch, _ = handles(s)
    rot = P.arkv_rotary(freq)
    q_out = torch.empty_like(s.q)
    P.arkv_paged_append(pages, batch, rot, s.q, kn, vn, pos, q_out)
    q2 = s.q.clone()
    P.arkv_paged_append(pages, batch, rot, q2, kn, vn, pos, q2)
    assert torch.equal(q2, q_out)
    v0 = s.v.clone()
    s.v[int(s.table[0, 0]), :, :3] = 0
    P.arkv_paged_append(pages, batch, rot, None, kn, vn, pos, None)
    assert torch.equal(s.v.nan_to_num(5.0), v0.nan_to_num(5.0))
    assert torch.equal(s.v[int(s.table[0, 0]), :, :3], vn[2:5].transpose(0, 1))       # tokens 0 and 1 have no slot
    s.weight = None
    P.arkv_paged_append(P.arkv_pages(s.k, s.v, s.pos), batch, rot, None, kn, vn, pos, None)


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("kv,keep,sink,recent", [
    ((1,), (1,), 4, 32), ((40, 7), (36, 36), 4, 32), ((300, 0, 1000), (100, 100, 100), 4, 32), ((2500, 1024, 1025), (700, 1024, 1), 0, 0),
    ((999, 333), (0, 50), 4, 8), ((500, 500), (20, -3), 30, 30), ((5000, 3000), (2500, 2999), 1, 7), ((9000,), (4500,), 4, 32)])
def test_evict(kv, keep, sink, recent, seed):
    s = R.problem("cuda", [BF, FP][seed % 2], 4, 2, [64, 128][seed % 2], [16, 64, 32][seed], (0,) * len(kv), kv, seed=50 + seed,
                  spare_pages=400)
    if seed == 1:                                      # few different weights: ties everywhere, signs, zeros, infinities, NaN
        pick = torch.tensor([0.0, -0.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 1e-40], device="cuda")
        s.weight = pick[torch.randint(0, 8, s.weight.shape, generator=torch.Generator().manual_seed(2)).cuda()].contiguous()
    if seed == 2:
        s.weight.zero_()
    max_keep = max(max(keep), 1)
    need = -(-max_keep // s.page)
    dst = torch.tensor(s.spare[:need * len(kv)], dtype=torch.int32, device="cuda").reshape(len(kv), need)
    ref, lens = R.evict(s, keep, sink, recent, max_keep)
    before = {n: getattr(s, n).clone() for n in ("k", "v", "pos", "weight")}
    pages, batch, ws = handles(s)
    ws[TICKETS:].fill_(0xFF)
    kept = torch.full((len(kv), 2, max_keep), 99, dtype=torch.int32, device="cuda")
    new_len = torch.full((len(kv),), 99, dtype=torch.int32, device="cuda")
    P.arkv_paged_evict(pages, batch, torch.tensor(keep, dtype=torch.int32, device="cuda"), dst, kept, new_len, sink=sink, recent=recent, workspace=ws)
    assert new_len.tolist() == lens
    assert torch.equal(kept.cpu(), ref)
    for name, old in before.items():
        want = old.clone()
        for b, m in enumerate(lens):
            for h in range(2):
                j = ref[b, h, :m].long().cuda()
                to = torch.arange(m, device="cuda")
                want[dst[b].long()[to // s.page], h, to % s.page] = old[s.table[b].long()[j // s.page], h, j % s.page]
        assert torch.equal(getattr(s, name).view(torch.uint8), want.view(torch.uint8)), name


@pytest.mark.parametrize("what", ["drawn", "few", "equal", "nan", "one digit"])
@pytest.mark.parametrize("kv,keep,announced", [
    ((9000, 4097, 300), (2000, 4096, 299), None), ((20000,), (5001,), 36864), ((40001, 5), (10000, 5), None), ((4096, 0), (1000, 50), 70000),
    ((36864,), (36000,), None)])
def test_evict_of_many_rows(kv, keep, announced, what):
    """Units whose rows several workgroups count, or that do not fit a workgroup's registers; the same workspace again and again."""
    s = R.problem("cuda", BF, 2, 2, 64, 64, (0,) * len(kv), kv, seed=61, spare_pages=len(kv) * (-(-max(keep) // 64)), width=1100)
    g = torch.Generator().manual_seed(5)
    if what == "few":
        s.weight = torch.tensor([0.0, 1.0, 2.0, math.inf]).cuda()[torch.randint(0, 4, s.weight.shape, generator=g).cuda()].contiguous()
    elif what == "one digit":                          # keys that differ in their lowest bits alone
        s.weight = 1.0 + torch.randint(0, 300, s.weight.shape, generator=g).float().cuda() * 2.0 ** -23
    elif what != "drawn":
        s.weight.fill_(0.0 if what == "equal" else math.nan)
    s.table[0, 3] = -1
    max_keep, need = max(keep), -(-max(keep) // 64)
    dst = torch.tensor(s.spare[:need * len(kv)], dtype=torch.int32, device="cuda").reshape(len(kv), need)
    ref, lens = R.evict(s, keep, 4, 32, max_keep)
    before = {n: getattr(s, n).clone() for n in ("k", "v", "pos", "weight")}
    pages, batch, ws = handles(s, max_kv=announced)
    ws[TICKETS:].fill_(0xFF)
    keep_dev = torch.tensor(keep, dtype=torch.int32, device="cuda")
    for _ in range(3):
        kept = torch.full((len(kv), 2, max_keep), 99, dtype=torch.int32, device="cuda")
        new_len = torch.full((len(kv),), 99, dtype=torch.int32, device="cuda")
        P.arkv_paged_evict(pages, batch, keep_dev, dst, kept, new_len, workspace=ws)
        assert new_len.tolist() == lens and torch.equal(kept.cpu(), ref)
        assert not ws[:TICKETS].any()
    for name, old in before.items():
        want = old.clone()
        for b, m in enumerate(lens):
            for h in range(2):
                j, to = ref[b, h, :m].long().cuda(), torch.arange(m, device="cuda")
                page = s.table[b].long()[j // 64]
                real = (page >= 0) & (page < s.n_pages)
                want[dst[b].long()[to // 64][real], h, (to % 64)[real]] = old[page[real], h, (j % 64)[real]]
        assert torch.equal(getattr(s, name).view(torch.uint8), want.view(torch.uint8)), name


def test_evict_around_absent_pages():
    s = R.problem("cuda", BF, 4, 2, 64, 16, (0,), (200,), seed=60, spare_pages=9)
    s.table[0, 2] = -1
    dst = torch.tensor([s.spare[:7]], dtype=torch.int32, device="cuda")
    dst[0, 1] = s.n_pages                              # nothing is written there
    k0 = s.k.clone()
    pages, batch, ws = handles(s)
    kept, lens = torch.empty((1, 2, 100), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    P.arkv_paged_evict(pages, batch, torch.tensor([100], dtype=torch.int32, device="cuda"), dst, kept, lens, workspace=ws)
    ref, _ = R.evict(s, [100], 4, 32, 100)
    assert torch.equal(kept.cpu(), ref) and not ((ref >= 32) & (ref < 48)).any()
    assert torch.equal(s.k[s.spare[0], 1], k0[s.table[0].long()[ref[0, 1, :16].cuda() // 16], 1, ref[0, 1, :16].long().cuda() % 16])


def test_other_streams_and_bitwise_repeats():
    s = R.problem("cuda", BF, 8, 2, 128, 16, (70, 1, 1), (3000, 5000, 10), seed=70)
    o1, l1 = attend(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, l2 = attend(s)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)
    pages, batch, ws = handles(s)
    w = []
    for _ in range(2):
        P.arkv_paged_weights(pages, batch, s.q, s.scale, l1, decay=0.0, workspace=ws)
        w.append(s.weight.clone())
    assert torch.equal(w[0].nan_to_num(5.0), w[1].nan_to_num(5.0))


def test_a_captured_step_follows_lengths_and_tables():
    """append, attention, weights, eviction in one graph, replayed with other lengths, pages and rows in the same arrays."""
    q, kv = (1, 40, 1), (500, 90, 33)
    s = R.problem("cuda", BF, 8, 2, 64, 16, q, kv, seed=71, spare_pages=60)
    pages = P.arkv_pages(s.k, s.v, s.pos, s.weight)
    batch = P.arkv_page_batch(s.cu_q, s.kv_len, s.table, s.n, 40, 512)
    ws = P.arkv_paged_workspace(pages, batch, s.hq)
    dst = torch.tensor(s.spare[:12], dtype=torch.int32, device="cuda").reshape(3, 4)
    keep = torch.tensor([60, 50, 64], dtype=torch.int32, device="cuda")
    kept, lens = torch.empty((3, 2, 64), dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).cuda()
    rot = P.arkv_rotary(freq)
    new = torch.randn(s.n, 12, 64, device="cuda").to(BF)
    positions = torch.arange(s.n, dtype=torch.int32, device="cuda")[None].contiguous()
    q_rot, out, lse = torch.empty(s.n, 8, 64, dtype=BF, device="cuda"), torch.empty(s.n, 8, 64, dtype=BF, device="cuda"), torch.empty(s.n, 8, device="cuda")

    def step():
        P.arkv_paged_append(pages, batch, rot, new[:, :8], new[:, 8:10], new[:, 10:], positions, q_rot)
        P.arkv_paged_attention(pages, batch, q_rot, s.scale, out, lse=lse, workspace=ws)
        P.arkv_paged_weights(pages, batch, q_rot, s.scale, lse, workspace=ws)
        P.arkv_paged_evict(pages, batch, keep, dst, kept, lens, workspace=ws)

    state = {n: getattr(s, n).clone() for n in ("k", "v", "pos", "weight")}
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, (cu, kvl) in enumerate([((0, 1, 41, 42), (500, 90, 33)), ((0, 0, 30, 42), (0, 64, 33)), ((0, 12, 13, 42), (499, 1, 31)), ((0, 1, 41, 42), (500, 90, 33))]):
        s.cu_q.copy_(torch.tensor(cu, dtype=torch.int32)); s.kv_len.copy_(torch.tensor(kvl, dtype=torch.int32))
        new.copy_(torch.randn(s.n, 12, 64, device="cuda"))
        got = []
        for run in (graph.replay, step):
            for name in state:
                getattr(s, name).copy_(state[name])
            run()
            torch.cuda.synchronize()
            got.append([x.clone() for x in (out, lse, kept, lens, s.k, s.weight, s.pos)])
        for a, b in zip(*got):
            assert torch.equal(a.float().nan_to_num(3.0), b.float().nan_to_num(3.0)), i


def test_the_example_equals_dense_attention_until_it_evicts():
    """Chunked prompts and single tokens through the example's layer against one dense causal attention per request."""
    from paper_2603_08727_amd.paged_example import PagedLayer
    torch.manual_seed(3)
    layer = PagedLayer(3, n_pages=128, limit=4000, budget=100, max_tokens=64)
    plan = [(64, 0, 5), (64, 40, 0), (1, 60, 1), (30, 1, 1), (1, 1, 1)]
    xs, ys = [[], [], []], [[], [], []]
    for q_len in plan:
        x = torch.randn(sum(q_len), 512, device="cuda").to(BF)
        y = layer.step(x, list(q_len))
        at = 0
        for r, a in enumerate(q_len):
            xs[r].append(x[at:at + a]); ys[r].append(y[at:at + a])
            at += a
    for r in range(3):
        x, y = torch.cat(xs[r]), torch.cat(ys[r])
        n = x.shape[0]
        assert layer.rows[r] == layer.seen[r] == n
        qkv = (x @ layer.w_qkv).view(n, 12, 64)
        positions = torch.arange(n, device="cuda")[None]
        q, k = (R.rotate(part, positions, layer.rotary.freq, [0] * 32, False)[0].to(BF).double() for part in (qkv[:, :8], qkv[:, 8:10]))
        v = qkv[:, 10:].double()
        out = torch.empty(n, 8, 64, dtype=torch.float64, device="cuda")
        for h in range(8):
            s = (q[:, h] @ k[:, h // 4].t()) / 8.0
            s = s.masked_fill(torch.ones_like(s).triu(1).bool(), -math.inf)
            out[:, h] = torch.softmax(s, -1) @ v[:, h // 4]
        ref = out.reshape(n, 512) @ layer.w_out.double()
        # stored roundings: rotated q and k (2^-9 of a logit each, at one rounding that falls the other way), probabilities, the
        # output, its projection: a few 2^-8 of the row's size
        assert float((y.double() - ref).norm() / ref.norm()) < 4 * 2.0 ** -8


def test_the_example_keeps_its_requests_within_their_budget():
    from paper_2603_08727_amd.paged_example import PagedLayer
    torch.manual_seed(4)
    layer = PagedLayer(2, n_pages=64, limit=96, budget=64, max_tokens=64)
    for step in range(30):
        q_len = [64, 0] if step < 3 else [1, 64] if step < 6 else [1, 1]
        y = layer.step(torch.randn(sum(q_len), 512, device="cuda").to(BF), q_len)
        assert torch.isfinite(y).all()
        assert all(n <= 96 for n in layer.rows)
        pages = layer.held[0] + layer.held[1] + layer.free
        assert sorted(pages) == list(range(64))        # no page is lost or held twice
    for r in range(2):
        for h in range(2):
            held = torch.tensor(layer.held[r], device="cuda").long()
            pos = layer.pages.pos[held, h].reshape(-1)[:layer.rows[r]]
            assert (pos[1:] > pos[:-1]).all() and int(pos[-1]) == layer.seen[r] - 1   # in order, the latest there
            assert pos[:4].tolist() == [0, 1, 2, 3]                                    # and the first four


def test_eviction_results_beside_its_lengths():
    """new_len and kept right behind kv_len and keep in one array: neighbours are no overlap, and the lengths stay as they are."""
    s = R.problem("cuda", BF, 8, 4, 64, 16, (0, 0, 0), (700, 90, 333), seed=80, spare_pages=30)
    line = torch.full((9 + 3 * 4 * 100,), 77, dtype=torch.int32, device="cuda")
    line[:3], line[6:9] = s.kv_len, torch.tensor([100, 80, 60], dtype=torch.int32, device="cuda")
    s.kv_len, new_len, keep, kept = line[:3], line[3:6], line[6:9], line[9:].view(3, 4, 100)
    pages, batch, ws = handles(s)
    dst = torch.tensor(s.spare[:21], dtype=torch.int32, device="cuda").reshape(3, 7)
    P.arkv_paged_evict(pages, batch, keep, dst, kept, new_len, workspace=ws)
    ref, lens = R.evict(s, [100, 80, 60], 4, 32, 100)
    assert new_len.tolist() == lens and torch.equal(kept.cpu(), ref)
    assert s.kv_len.tolist() == [700, 90, 333] and keep.tolist() == [100, 80, 60]
    for bad in (dict(new_len=s.kv_len), dict(new_len=keep), dict(kept=line[:1200].view(3, 4, 100))):
        with pytest.raises(P.ArkvError) as e:
            P.arkv_paged_evict(pages, batch, keep, dst, bad.get("kept", kept), bad.get("new_len", new_len), workspace=ws)
        assert e.value.code == P.EINVAL


def test_a_workspace_for_the_largest_bounds_serves_every_call():
    """Sized once for more sequences, tokens and rows than any of the batches has; single tokens and short chunks are cut finer."""
    g = dict(dtype=BF, hq=8, hkv=2, d=128, page=16)
    batches = [((600,) * 2, (4000, 2100)), ((1,), (6000,)), ((1,) * 12, (3000,) * 12), ((64,), (6000,)), ((20, 1, 1), (5000, 6000, 4000)), ((300,), (6000,))]
    problems = [R.problem("cuda", q_len=q, kv_len=kv, seed=90 + i, **g) for i, (q, kv) in enumerate(batches)]
    s = problems[0]
    limits = P.arkv_page_batch(torch.zeros(13, dtype=torch.int32, device="cuda"), torch.zeros(12, dtype=torch.int32, device="cuda"),
                               torch.zeros(12, 375, dtype=torch.int32, device="cuda"), 1200, 600, 6000)
    ws = P.arkv_paged_workspace(P.arkv_pages(s.k, s.v, s.pos, s.weight), limits, 8)
    for s in problems:
        want, want_lse = attend(s)
        pages, batch, _ = handles(s)
        ws[TICKETS:].fill_(0xFF)
        out, lse = torch.empty_like(want), torch.empty_like(want_lse)
        P.arkv_paged_attention(pages, batch, s.q, s.scale, out, lse=lse, workspace=ws)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        ref, tol = R.weights(s, lse, 0.5, s.weight)
        ws[TICKETS:].fill_(0xFF)
        P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.5, workspace=ws)
        R.close(s.weight, ref, tol, "weight")
        assert not ws[:TICKETS].any()


@pytest.mark.parametrize("q,kv,hq,hkv", [
    ((1, 40, 0, 2) * 40, (5000, 70, 0, 300) + (33, 100, 9, 2100) * 39, 16, 8),      # 1280 units: too many for tickets, three pieces
    ((1, 300, 2) * 45, (17000, 300, 2) + (64, 700, 2500) * 44, 8, 8),               # nine pieces
    ((1100, 1, 1, 2), (1100, 40000, 33000, 2049), 16, 16),                          # more than sixteen, beside a chunk that is joined
    ((17, 1, 0), (40000, 36000, 70), 2, 1)])                                        # both kinds of rows in many pieces
def test_rows_of_split_sequences_are_joined_in_a_launch(q, kv, hq, hkv):
    s = R.problem("cuda", BF, hq, hkv, 64, 16, q, kv, seed=17, extra_tokens=3)
    check_attention(s)
    check_attention(s, prefix=torch.tensor([t - a // 2 for a, t in zip(q, kv)], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("kv,keep", [(200, 130), (9000, 8700)])
def test_rows_without_a_number_and_absent_rows_rank_alike(kv, keep):
    """Both lie below every number, -infinity too, and among themselves the lower slot stays first."""
    s = R.problem("cuda", BF, 2, 2, 64, 16, (0,), (kv,), seed=81, spare_pages=-(-keep // 16))
    held = s.table[0].long()
    s.weight[held] = torch.where(torch.rand(s.weight[held].shape, generator=torch.Generator().manual_seed(8)).cuda() < 0.5, math.nan, -math.inf)
    s.table[0, 4] = -1                                 # slots 64 to 79, NaN before and behind them
    dst = torch.tensor([s.spare], dtype=torch.int32, device="cuda")
    pages, batch, ws = handles(s)
    kept, lens = torch.empty((1, 2, keep), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    P.arkv_paged_evict(pages, batch, torch.tensor([keep], dtype=torch.int32, device="cuda"), dst, kept, lens, workspace=ws)
    for h in range(2):
        w = R.rows(s, s.weight, 0, h)[0]
        number = ~torch.isnan(w)
        number[64:80] = False
        middle = torch.arange(4, kv - 32, device="cuda")
        order = torch.cat([middle[number[4:kv - 32]], middle[~number[4:kv - 32]]])[:keep - 36]
        want = torch.cat([torch.arange(4, device="cuda"), order.sort().values, torch.arange(kv - 32, kv, device="cuda")])
        assert torch.equal(kept[0, h].long(), want)


@pytest.mark.parametrize("cap", [257.0, 3000.0, 1e5, 1e9, 3e38])
@pytest.mark.parametrize("q,kv", [((1, 2), (700, 40)), ((60, 130), (800, 400))])
@pytest.mark.parametrize("dtype,d,far", [(BF, 128, False), (FP, 64, True)])
def test_wide_caps_do_not_drown_the_logits(dtype, d, far, q, kv, cap, monkeypatch):
    """The wider the cap, the nearer the uncapped scores: off by 2^-19 of a logit, not by a share of the cap."""
    plain = R.logits

    def logits(s, b, hq, cap=0.0, **kw):
        x, err = plain(s, b, hq, cap, **kw)
        bare = plain(s, b, hq)[0]
        return x, plain(s, b, hq, **kw)[1] + 2.0 ** -19 * float(bare[torch.isfinite(bare)].abs().max())

    monkeypatch.setattr(R, "logits", logits)
    s = R.problem("cuda", dtype, 8, 2, d, 16, q, kv, seed=18, hot=20.0)
    kw = dict(cap=cap)
    if far:
        kw["slopes"], kw["q_pos"] = slopes_of(s)
    _, lse = check_attention(s, **kw)
    pages, batch, ws = handles(s)
    ref, tol = R.weights(s, lse, 1.0, s.weight, **kw)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, workspace=ws, **kw)
    R.close(s.weight, ref, tol, "weight")


@pytest.mark.parametrize("kw", [dict(sink=1 << 32), dict(recent=(1 << 32) + 8), dict(sink=-(1 << 32))])
def test_evictions_whose_numbers_do_not_fit_32_bits_are_refused(kw):
    s = R.problem("cuda", BF, 2, 2, 64, 16, (0,), (100,), seed=82, spare_pages=4)
    pages, batch, ws = handles(s)
    kept, lens = torch.full((1, 2, 50), 9, dtype=torch.int32, device="cuda"), torch.full((1,), 9, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="32 bits"):
        P.arkv_paged_evict(pages, batch, torch.tensor([50], dtype=torch.int32, device="cuda"), torch.tensor([s.spare], dtype=torch.int32, device="cuda"),
                           kept, lens, workspace=ws, **kw)
    assert (kept == 9).all() and int(lens) == 9


def test_a_refused_step_of_the_example_changes_nothing():
    """Out of pages for the rows, or for the eviction behind them, or too many tokens: the next step goes on as if it had not been tried."""
    from paper_2603_08727_amd.paged_example import PagedLayer
    layers = [PagedLayer(2, n_pages=12, limit=96, budget=64, max_tokens=64) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(5)

    def rows(n):
        return torch.randn(n, 512, generator=g, device="cuda").to(BF)

    for q_len, bad in [([60, 20], [(RuntimeError, [64, 64])]),         # 14 pages for the rows alone
                       ([30, 30], [(RuntimeError, [64, 1]), (ValueError, [65, 0]), (ValueError, [1]), (ValueError, [2, -1])]),
                       ([1, 1], [(RuntimeError, [10, 1])])]:           # 101 rows have their pages, but not the 4 to cut them into
        x = rows(sum(q_len))
        want = layers[0].step(x, list(q_len))
        assert torch.equal(layers[1].step(x, list(q_len)), want)
        for error, refused in bad:
            state = [str(getattr(layers[1], n)) for n in ("free", "held", "rows", "seen")] + [layers[1].table.clone(), layers[1].pages.k.clone()]
            with pytest.raises(error):
                layers[1].step(rows(max(0, sum(refused))), refused)
            assert state[:4] == [str(getattr(layers[1], n)) for n in ("free", "held", "rows", "seen")]
            assert torch.equal(state[4], layers[1].table) and torch.equal(state[5], layers[1].pages.k)
    x = rows(2)
    assert torch.equal(layers[0].step(x, [1, 1]), layers[1].step(x, [1, 1]))


def ragged(chunks, many):
    """130 sequences: single tokens and a chunk now and then, empty ones and absent ones around the 64th and the 128th."""
    q = [0 if b in (0, 62, 64, 127) else chunks[b % len(chunks)] if b in (1, 61, 63, 65, 100, 126, 128, 129) else 1 for b in range(130)]
    kv = [0 if b in (64, 101) else a + 5 + 37 * b % 211 for b, a in enumerate(q)]
    if many:
        kv[3], kv[66], kv[129] = 17001, 3000, 2500     # nine pieces: joined by a launch
    return q, kv


@pytest.mark.parametrize("chunks,many", [((2, 40, 150), False), ((3, 1, 300), True), ((1, 2), False), ((2,), True)])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 16, 8, 64), (FP, 6, 2, 128)])
def test_batches_of_more_than_64_sequences(dtype, hq, hkv, d, chunks, many):
    """Searches for a token's sequence go round more than once, in append, attention and its joins; weights of all sequences."""
    q, kv = ragged(chunks, many)
    s = R.problem("cuda", dtype, hq, hkv, d, 16, q, kv, seed=83, extra_tokens=2, fused=True)
    s.table[5, 0] = -1
    g = torch.Generator().manual_seed(6)
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).cuda()
    positions = torch.randint(0, 100000, (1, s.n), generator=g, dtype=torch.int32).cuda()
    new = torch.randn(s.n, 2 * hkv, d, generator=g).to(dtype).cuda()
    pages, batch, ws = handles(s)
    want = {n: getattr(s, n).clone() for n in ("k", "v", "pos", "weight")}
    q_out = torch.full((s.n, hq, d), 7.0, dtype=dtype, device="cuda")
    P.arkv_paged_append(pages, batch, P.arkv_rotary(freq), s.q, new[:, :hkv], new[:, hkv:], positions, q_out)
    n = sum(q)
    check_append(s, want, new[:, :hkv], new[:, hkv:], positions, freq, [0] * (d // 2), False, q_out)
    assert (q_out[n:] == 7).all()
    _, lse = check_attention(s)
    ref, tol = R.weights(s, lse, 0.5, s.weight)
    P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.5, workspace=ws)
    R.close(s.weight, ref, tol, "weight")


def check_append(s, before, kn, vn, positions, freq, axis, adjacent, q_out):
    """Turned queries, and pools that differ from `before` in the new tokens' slots alone."""
    n = sum(s.q_len)
    (rq, tq), (rk, tk) = (R.rotate(x[:n], positions[:, :n], freq, axis, adjacent) for x in (s.q, kn))
    R.close(q_out[:n], rq, tq, "q")
    b = torch.repeat_interleave(torch.arange(s.B), torch.tensor(s.q_len))
    i = torch.cat([torch.arange(a) for a in s.q_len])
    slot = (torch.tensor(s.kv_len_list) - torch.tensor(s.q_len))[b] + i
    page = s.table.cpu()[b, slot.clamp(min=0) // s.page].long()
    there = (slot >= 0) & (page >= 0) & (page < s.n_pages)
    t, page, off = torch.arange(n)[there].cuda(), page[there].cuda(), (slot[there] % s.page).cuda()
    R.close(s.k[page, :, off], rk[t], tk[t], "k")
    before["k"][page, :, off] = s.k[page, :, off]
    before["v"][page, :, off] = vn[t]
    before["pos"][page, :, off] = positions[0, t][:, None].expand(-1, s.hkv)
    before["weight"][page, :, off] = 0.0
    for name, want in before.items():
        assert torch.equal(getattr(s, name).view(torch.uint8), want.view(torch.uint8)), name


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("q,kv", [((1,) * 16, tuple(range(1, 1600, 100))), ((5, 11), (5, 900)), ((2100,), (2131,)), ((700, 1400, 3), (700, 1500, 40))])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 32, 8, 128), (FP, 40, 5, 64), (BF, 64, 8, 128)])
def test_appends_whose_tokens_are_several_waves_or_rounds(dtype, hq, hkv, d, q, kv, adjacent):
    """Few tokens are dealt out over waves by their heads, many (from 2048 on) are one wave's each, in several rounds."""
    s = R.problem("cuda", dtype, hq, hkv, d, 16, q, kv, seed=84, fused=True)
    g = torch.Generator().manual_seed(7)
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).cuda()
    axis = [i % 3 for i in range(d // 2)]
    positions = torch.randint(0, 1 << 20, (3, s.n), generator=g, dtype=torch.int32).cuda()
    new = torch.randn(s.n, 2 * hkv, d, generator=g).to(dtype).cuda()
    want = {n: getattr(s, n).clone() for n in ("k", "v", "pos", "weight")}
    pages, batch, _ = handles(s)
    q_out = torch.empty((s.n, hq, d), dtype=dtype, device="cuda")
    P.arkv_paged_append(pages, batch, P.arkv_rotary(freq, axis, 3, adjacent), s.q, new[:, :hkv], new[:, hkv:], positions, q_out)
    check_append(s, want, new[:, :hkv], new[:, hkv:], positions, freq, axis, adjacent, q_out)


@pytest.mark.parametrize("q,d,page", [(1, 64, 64), (1, 128, 16), (4, 64, 16)])
@pytest.mark.parametrize("far", [False, True])
def test_weights_of_many_rows_per_wave(q, d, page, far):
    """16 x 8 units of thousands of rows: five to nine tiles a wave, lengths that end inside one, absent pages."""
    kv = [9001 if d == 64 else 5003] + [4000 + 331 * b for b in range(14)] + [70]
    s = R.problem("cuda", BF, 32, 8, d, page, (q,) * 16, kv, seed=85)
    s.table[1, 7], s.table[2, 30] = -1, s.n_pages
    kw = {}
    if far:
        kw["slopes"], kw["q_pos"] = slopes_of(s)
    _, lse = attend(s, **kw)
    pages, batch, ws = handles(s)
    for decay, other in [(0.75, False), (1.0, True), (0.0, False)]:
        carried = torch.rand_like(s.weight) if other else s.weight.clone()
        ref, tol = R.weights(s, lse, decay, carried, **kw)
        P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=decay, carried=carried if other else None, workspace=ws, **kw)
        R.close(s.weight, ref, tol, "weight")


@pytest.mark.parametrize("n,h", [(1, 8), (5, 1), (1, 1)])
def test_strides_of_a_single_token_or_head_do_not_matter(n, h):
    """torch gives such axes any stride: here 1, which no row could have."""
    s = R.problem("cuda", BF, h, 1, 64, 16, (n,), (90,), seed=86)
    new = torch.randn(n, 1, 64, device="cuda").to(BF)
    q, out = s.q, []
    for odd in (False, True):
        if odd:
            strides = (1 if n == 1 else q.stride(0), 1 if h == 1 else q.stride(1), 1)
            s.q, new = q.as_strided(q.shape, strides), new.as_strided(new.shape, (1 if n == 1 else 64, 1, 1))
        pages, batch, ws = handles(s)
        turned = torch.empty_like(q)
        P.arkv_paged_append(pages, batch, P.arkv_rotary(None), s.q, new, new, torch.arange(n, dtype=torch.int32, device="cuda")[None].contiguous(), turned)
        o, lse = check_attention(s)
        P.arkv_paged_weights(pages, batch, s.q, s.scale, lse, decay=0.0, workspace=ws)
        out.append([turned, o, lse, s.k.nan_to_num(5.0), s.weight.nan_to_num(5.0)])
        out[-1] = [x.clone() for x in out[-1]]
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("what", [math.nan, 40.0])
@pytest.mark.parametrize("q,kv", [((2,), (8190,)), ((4,), (20001,)), ((40,), (5000,))])
def test_rows_are_independent_to_the_bit(q, kv, what, dtype):
    """A key that the last token alone sees, in a tile behind a wave's first: the rounding of the other tokens' rows does not change either."""
    s = R.problem("cuda", dtype, 8, 2, 64, 16, q, kv, seed=87)
    clean, clean_lse = attend(s)
    last = kv[0] - 1
    s.k[int(s.table[0, last // 16]), :, last % 16] = what if what != what else s.q[-1, ::4] * what
    out, lse = attend(s)
    assert not torch.equal(out[-1], clean[-1])
    assert torch.equal(out[:-1], clean[:-1]) and torch.equal(lse[:-1], clean_lse[:-1])
