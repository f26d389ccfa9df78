"""GPU tests of the kernel for blocks of 128 rows over packed pages, under a window and for drafted trees (calls that are divided into groups of
16 rows are test_gpu_packed.py's): every way to cut and to join, scores, absent pages, hidden rows, values that are no numbers, rows without
a slot.  Each test says which way the call has to go."""
import math

import pytest
import torch

from paper_2603_08727_amd import paged as P
import packed_ref as K
import paged_ref as R
import sight_ref as S
from test_gpu_packed import attend, handles, scores_of

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
NO, LAUNCH, BLOCKS, ROWS = range(4)                    # who joins the pieces of a block


def problem(bits, dtype, hq, hkv, d, q, kv, seed=0, page=16, **kw):
    make = dict(hq=hq, hkv=hkv, d=d, page=page, q_len=q, kv_len=kv, seed=seed, **kw)
    return R.problem("cuda", dtype, **make) if bits == 16 else K.problem("cuda", bits, dtype, **make)


def check(s, window=0, sink=0, tree=None, few=None, join=None, pieces=None, **kw):
    cut = S.cut(s, window, sink, tree, **kw)
    assert cut.blocks and not cut.groups and few in (None, cut.few) and join in (None, cut.join) and pieces in (None, cut.pieces), vars(cut)
    out, lse = attend(s, window, sink, tree, **kw)
    ref, rl, tol, ltol = S.attention(s, window, sink, tree, **kw)
    n = sum(s.q_len)
    R.close(out[:n], ref[:n], tol[:n], "out")
    R.close(lse[:n], rl[:n], ltol[:n], "lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    again = attend(s, window, sink, tree, **kw)
    assert torch.equal(torch.nan_to_num(out, 9.0), torch.nan_to_num(again[0], 9.0)) and torch.equal(lse.nan_to_num(9.0), again[1].nan_to_num(9.0))
    return out, lse


# all of the same length: blocks alone; some tokens beside them
ALONE, BESIDE = ((512, 512), (2048, 2000)), ((400, 1, 700), (3000, 900, 2500))


@pytest.mark.parametrize("kind", ["", "cap", "wide", "distance", "prefix", "cap+distance+prefix"])
@pytest.mark.parametrize("q,kv", [ALONE, BESIDE])
@pytest.mark.parametrize("bits,dtype,hq,hkv,d,window", [(8, BF, 8, 2, 128, 0), (8, FP, 8, 2, 64, 0), (4, BF, 12, 4, 64, 0), (4, FP, 4, 4, 128, 0), (16, BF, 8, 2, 128, 1000),
                                                        (16, FP, 12, 4, 64, 1000), (8, FP, 16, 1, 64, 1000), (4, BF, 8, 1, 128, 1000)])
def test_scores(bits, dtype, hq, hkv, d, window, q, kv, kind):
    s = problem(bits, dtype, hq, hkv, d, q, kv, seed=d + len(kind), hot=6.0, extra_tokens=len(q) - 2)
    kw = dict(cap=300.0) if kind == "wide" else scores_of(kind, s, q, kv)
    check(s, window, 4 if window else 0, few=len(q) == 3, **kw)


# (shape, window, sink, heads, channels, and where they are of packed rows: who joins, the most pieces)
WINDOWS = [((512, 512), (2048, 2000), 300, 4, 16, 1, 64, LAUNCH, 2), ((2100,), (2100,), 300, 40, 8, 2, 128, LAUNCH, 2), ((2100,), (4000,), 1000, 0, 8, 2, 128, LAUNCH, 3),
           ((2100,), (4000,), 1000, 4, 8, 2, 64, BLOCKS, 5), ((900, 30, 1), (5000, 100, 3000), 1000, 4, 12, 4, 64, BLOCKS, 5),
           ((2100,), (2100,), 300, 4, 16, 1, 64, NO, 1), ((2100,), (3500,), 1600, 17, 32, 8, 128, NO, 1), ((1200,), (6000,), 1000, 1, 16, 1, 64, BLOCKS, 5)]


@pytest.mark.parametrize("bits,dtype", [(16, BF), (16, FP), (8, BF), (8, FP), (4, BF), (4, FP)])
@pytest.mark.parametrize("q,kv,window,sink,hq,hkv,d,join,pieces", WINDOWS)
def test_windows(q, kv, window, sink, hq, hkv, d, join, pieces, bits, dtype):
    s = problem(bits, dtype, hq, hkv, d, q, kv, seed=window + sink, page=32)
    check(s, window, sink, join=join)


@pytest.mark.parametrize("bits,dtype", [(8, BF), (8, FP), (4, BF), (4, FP)])
@pytest.mark.parametrize("q,kv,hq,hkv,d,join", [((2100,), (3500,), 32, 8, 128, NO), ((512, 512), (2048, 2000), 8, 2, 128, LAUNCH), ((600, 600), (1500, 600), 8, 1, 128, LAUNCH),
                                                ((2100,), (2100,), 8, 2, 64, BLOCKS), ((1200,), (6000,), 4, 4, 128, BLOCKS), ((2000,), (2100,), 32, 8, 64, None)])
def test_causal_chunks_of_packed_rows(q, kv, hq, hkv, d, join, bits, dtype):
    check(problem(bits, dtype, hq, hkv, d, q, kv, seed=sum(q), page=64, fused=True), join=join)


@pytest.mark.parametrize("window,sink", [(0, 0), (1000, 4), (30, 0)])
@pytest.mark.parametrize("bits,dtype,hq,hkv,d", [(16, BF, 8, 2, 128), (16, FP, 12, 4, 64), (8, BF, 8, 2, 64), (4, FP, 8, 1, 128)])
@pytest.mark.parametrize("q,kv", [ALONE, BESIDE])
def test_trees(q, kv, bits, dtype, hq, hkv, d, window, sink):
    """Hundreds of drafts: words of many, and windows that end within them."""
    s = problem(bits, dtype, hq, hkv, d, q, kv, seed=sum(q) + window)
    cut = S.cut(s, window, sink, K.drafts(s, seed=1))
    if not cut.blocks:                                 # (a short window's rows are few enough for groups)
        assert window == 30
        s = problem(bits, dtype, hq * 4, hkv * 4, d, q, kv, seed=sum(q) + window)
    check(s, window, sink, K.drafts(s, seed=1))


@pytest.mark.parametrize("bits,dtype", [(16, BF), (8, BF), (8, FP), (4, FP)])
@pytest.mark.parametrize("window,sink", [(0, 0), (900, 4)])
def test_trees_of_eight_requests(window, sink, bits, dtype):
    q, kv = (64, 25, 40, 33, 64, 1, 50, 61), (2000, 1500, 700, 1999, 64, 1300, 1000, 1203)
    s = problem(bits, dtype, 32, 8, 128, q, kv, seed=window, extra_tokens=3)
    check(s, window, sink, K.drafts(s, seed=2), few=True)


@pytest.mark.parametrize("bits", [16, 8])
def test_any_bits_are_a_tree(bits):
    q, kv = (512, 500), (512, 2000)
    s = problem(bits, BF, 8, 2, 64, q, kv, seed=2)
    tree = torch.rand(s.n, 512, generator=torch.Generator().manual_seed(3)) < 0.3
    tree[0] = False
    out, lse = check(s, 0, 0, tree)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    check(s, 1200, 2, tree)
    check(s, 0, 0, tree, **scores_of("cap+distance+prefix", s, q, kv))


@pytest.mark.parametrize("bits,window", [(8, 0), (4, 0), (16, 1000), (8, 1000)])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (12, 4, 64)])
def test_absent_pages(hq, hkv, d, bits, window):
    q, kv = BESIDE
    s = problem(bits, BF, hq, hkv, d, q, kv, seed=4)
    for b, at, page in [(0, 0, -1), (0, 5, s.n_pages), (0, 6, 2 ** 31 - 1), (0, 150, -1), (0, 187, -1), (2, 2, -2 ** 31), (2, 140, -5), (2, 113, s.n_pages)]:
        s.table[b, at] = page
    check(s, window, 20)
    s.table[2] = -1
    out, lse = check(s, window, 20)
    assert (lse[401:] == -math.inf).all() and (out[401:] == 0).all()


@pytest.mark.parametrize("bits,window", [(8, 0), (4, 0), (16, 1000), (8, 1000), (4, 1000)])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("q,kv", [ALONE, BESIDE])
def test_rows_that_are_no_numbers(q, kv, hq, hkv, d, bits, window):
    """Values that are no numbers in rows that some tokens see, in several tiles and both halves of a tile: those tokens have them, the others' results
    are as they were, to the bit; then keys."""
    s = problem(bits, BF, hq, hkv, d, q, kv, seed=5)
    clean, clean_lse = check(s, window, 4 if window else 0)
    see = S.sight(s, 0, None, window, 4 if window else 0)
    sees = torch.zeros(q[0], dtype=torch.bool, device="cuda")
    slots = [kv[0] - 1, kv[0] - 2, kv[0] - q[0] // 2, kv[0] - q[0] // 2 - 33, kv[0] - q[0] // 2 - 60] + ([kv[0] - q[0] - window + 100] if window else [])
    for n, slot in enumerate(slots):
        page, off = int(s.table[0, slot // 16]), slot % 16
        for h, ch in ((0, 3), (hkv - 1, 40)):
            if bits == 16:
                s.v[page, h, off, ch] = math.nan if n % 2 else math.inf
            else:
                K.set_value(s, "v", page, h, off, ch)
        sees |= see[:, slot]
    assert 0 < int(sees.sum()) < q[0]
    out, lse = check(s, window, 4 if window else 0)
    keep = torch.ones(s.n, dtype=torch.bool, device="cuda")
    keep[:q[0]] = ~sees
    assert torch.equal(out[keep], clean[keep]) and torch.equal(lse, clean_lse)
    for slot in slots:
        page, off = int(s.table[0, slot // 16]), slot % 16
        if bits == 16:
            s.k[page, :, off] = math.nan
        else:
            s.k_scale[page, :, off] = 255
    out, lse = attend(s, window, 4 if window else 0)
    assert torch.equal(out[keep], clean[keep]) and torch.equal(lse[keep], clean_lse[keep])
    assert torch.isnan(out[:q[0]][sees]).all() and torch.isnan(lse[:q[0]][sees]).all()


@pytest.mark.parametrize("bits,dtype,hq,hkv,d", [(16, BF, 8, 2, 128), (16, FP, 8, 2, 64), (8, BF, 8, 2, 64), (4, BF, 12, 4, 128)])
@pytest.mark.parametrize("window", [0, 1000])
def test_rows_without_a_slot_see_nothing(window, bits, dtype, hq, hkv, d):
    if bits == 16 and not window:
        window = 1400
    q, kv = (2100, 3, 600), (1500, 40, 590)
    s = problem(bits, dtype, hq, hkv, d, q, kv, seed=3)
    out, lse = check(s, window, 2)
    for at, lost in ((0, 600), (2103, 10)):
        assert (out[at:at + lost] == 0).all() and (lse[at:at + lost] == -math.inf).all()
    check(s, window, 2, prefix=torch.tensor([1, 0, 30], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("window,sink,d", [(300, 20, 128), (1000, 20, 64)])
def test_what_a_window_hides_has_no_influence(window, sink, d, bits):
    """Neither rows nor table entries in front of the first token's window."""
    q, kv = (2100,), (4000,)
    s = problem(bits, BF, 8, 2, d, q, kv, seed=6)
    out, lse = check(s, window, sink)
    first = (kv[0] - q[0] - window + 1) // 16
    assert first > 2
    s.table[0, 2:first] = torch.tensor([-1, s.n_pages, 2 ** 30] * 100, dtype=torch.int32)[:first - 2].cuda()
    for j in list(range(sink, 32)) + list(range(16 * first, kv[0] - q[0] - window + 1)):
        page = int(s.table[0, j // 16])
        if bits == 16:
            s.k[page, :, j % 16], s.v[page, :, j % 16] = math.nan, math.inf
        else:
            s.k_scale[page, :, j % 16], s.v_scale[page, :, j % 16] = 255, 255
    again = attend(s, window, sink)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def loosely(s, window, sink, tree, max_q, max_kv, few=None, join=None, **kw):
    """A call whose bounds are looser than the lengths."""
    cut = S.cut(s, window, sink, tree, max_q=max_q, max_kv=max_kv, **kw)
    assert cut.blocks and not cut.groups and few in (None, cut.few) and join in (None, cut.join), vars(cut)
    pages, batch, ws = handles(s, max_q, max_kv)
    ws[1 << 16:].fill_(0xFF)
    out = torch.full((s.n, s.hq, s.d), 7.0, dtype=s.dtype, device="cuda")
    lse = torch.full((s.n, s.hq), 7.0, device="cuda")
    words = None
    if tree is not None:
        wide = torch.zeros(s.n, -(-max_q // 64) * 64, dtype=torch.bool)
        wide[:, :tree.shape[1]] = tree
        words = K.words(wide).cuda()
    sight = P.arkv_sight(window, sink, words) if window or tree is not None else None
    if hasattr(s, "bits"):
        P.arkv_packed_attention(pages, batch, s.q, s.scale, out, lse=lse, sight=sight, workspace=ws, **kw)
    else:
        P.arkv_paged_attention_sight(pages, batch, sight, s.q, s.scale, out, lse=lse, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert not ws[:1 << 16].any()
    ref, rl, tol, ltol = S.attention(s, window, sink, tree, **kw)
    n = sum(s.q_len)
    R.close(out[:n], ref[:n], tol[:n], "out")
    R.close(lse[:n], rl[:n], ltol[:n], "lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()


# Many short sequences beside few rows each: so many pieces, by their bounds, that rows are joined one by one, of few pieces and of many.
@pytest.mark.parametrize("bits,dtype,drafted,window", [(8, BF, False, 0), (4, FP, False, 0), (16, BF, True, 0), (8, FP, True, 9000), (16, FP, False, 9000), (4, BF, False, 3000)])
@pytest.mark.parametrize("hq,hkv,d,max_kv", [(1, 1, 64, 16384), (8, 8, 64, 16384), (4, 2, 128, 20000)])
def test_pieces_of_rows_are_joined(hq, hkv, d, max_kv, bits, dtype, drafted, window):
    q = [20 + b % 3 if b % 10 else 1 for b in range(100)]
    kv = [max(a, 301 * b % 4001) if b % 9 == 0 else a + b for b, a in enumerate(q)]
    kv[99] = 15000 if window else kv[99]
    s = problem(bits, dtype, hq, hkv, d, q, kv, seed=8, width=-(-max_kv // 16), extra_tokens=1)
    loosely(s, window, 4 if window else 0, K.drafts(s) if drafted else None, 30, max_kv, join=ROWS if (hq, max_kv) == (1, 16384) and window != 3000 else None)


@pytest.mark.parametrize("bits,window,drafted", [(16, 2600, False), (16, 0, True), (8, 0, False), (8, 2600, True), (4, 0, False)])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64)])
def test_bounds_may_be_loose(hq, hkv, d, bits, window, drafted):
    q, kv = (300, 2, 150), (5000, 700, 151)
    s = problem(bits, BF, hq, hkv, d, q, kv, seed=4, width=600, extra_tokens=400)
    loosely(s, window, 4 if window else 0, K.drafts(s) if drafted else None, s.n, 9600)


@pytest.mark.parametrize("bits,window", [(8, 0), (4, 500), (16, 500)])
def test_batches_of_more_than_64_sequences(bits, window):
    q = [1 if b % 3 else 150 + b % 5 for b in range(130)]
    q[40] = q[129] = 0
    kv = [max(a, 97 * b % 900) for b, a in enumerate(q)]
    check(problem(bits, BF, 8, 2, 64, q, kv, seed=5), window, 2, few=True)


@pytest.mark.parametrize("bits,d", [(8, 128), (4, 64), (16, 128)])
def test_a_captured_chunk_follows_lengths_tables_and_rows(bits, d):
    """One graph, whose kernel chooses its pieces by the lengths of each replay."""
    hq, hkv, B, most, max_kv = 8, 2, 4, 600, 4096
    width = max_kv // 16
    s = problem(bits, BF, hq, hkv, d, (1,) * B, (max_kv,) * B, seed=7)
    n = B * most
    s.q = torch.zeros(n, hq, d, dtype=BF, device="cuda")
    s.n, s.table = n, s.table[:, :width].contiguous()
    window = 900 if bits == 16 else 0
    pages, batch, ws = handles(s, most, max_kv)
    sight = P.arkv_sight(window, 4) if window else None
    out, lse = torch.zeros(n, hq, d, dtype=BF, device="cuda"), torch.zeros(n, hq, device="cuda")

    def step():
        if bits == 16:
            P.arkv_paged_attention_sight(pages, batch, sight, s.q, s.scale, out, lse=lse, workspace=ws)
        else:
            P.arkv_packed_attention(pages, batch, s.q, s.scale, out, lse=lse, sight=sight, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(0)
    lengths = set()
    for turn, (q, kv) in enumerate([((600, 600, 600, 600), (4096, 700, 4000, 3000)), ((1, 0, 500, 20), (4096, 5, 600, 4000)), ((16, 300, 1, 1), (16, 300, 4096, 1)),
                                    ((600, 1, 1, 1), (600, 4096, 4096, 4096)), ((599, 600, 17, 333), (4095, 601, 4001, 3003))]):
        s.q_len, s.kv_len_list = list(q), list(kv)
        s.cu_q.copy_(torch.tensor([sum(q[:b]) for b in range(B + 1)], dtype=torch.int32))
        s.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        s.table.copy_(s.table[torch.randperm(B, generator=g).cuda()])
        s.q.copy_(torch.randn(n, hq, d, generator=g).to(BF))
        cut = S.cut(s, window, 4 if window else 0, max_q=most, max_kv=max_kv)
        assert cut.blocks and not cut.groups
        lengths.add(cut.piece)
        results = []
        for run in (graph.replay, step):
            out.fill_(3.0)
            lse.fill_(3.0)
            run()
            torch.cuda.synchronize()
            results.append((out.clone(), lse.clone()))
        assert all(torch.equal(a, b) for a, b in zip(*results))
        ref, rl, tol, ltol = S.attention(s, window, 4 if window else 0)
        used = sum(q)
        R.close(out[:used], ref[:used], tol[:used], "out")
        R.close(lse[:used], rl[:used], ltol[:used], "lse")
        assert (out[used:] == 3).all() and (lse[used:] == 3).all()
    assert window or len(lengths) > 1


def test_another_stream_repeats_to_the_bit():
    s = problem(4, BF, 8, 2, 64, *BESIDE, seed=3)
    tree = K.drafts(s)
    first = check(s, 1000, 4, tree)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        second = attend(s, 1000, 4, tree)
    torch.cuda.synchronize()
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
