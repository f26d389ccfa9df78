"""CPU checks of how attention over packed pages, under a window or for drafted trees, is divided, and of the tests' matrices of what tokens see."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2603_08727_amd import binding as A
from paper_2603_08727_amd import paged as P
import packed_ref as K
import sight_ref as S


def cut(q, kv, hq, hkv, d, bits, window=0, sink=0, tree=False, n_tokens=None, max_q=None, max_kv=None, **kw):
    return S.Cut(P.arkv_debug_attention_cut(np.cumsum([0, *q]), kv, n_tokens or sum(q), max_q or max(q), max_kv or max(kv), hq, hkv, d, bits, window, sink,
                                            -(-(max_q or max(q)) // 64) if tree else 0, **kw))


def test_what_is_seen_is_the_same_as_whole_matrices():
    g = torch.Generator().manual_seed(1)
    pick = lambda hi: int(torch.randint(0, hi, (1,), generator=g))  # noqa: E731
    for _ in range(300):
        q = [pick(9) for _ in range(3)]
        kv = [pick(40) for _ in range(3)]
        s = K.R.problem("cpu", hq=2, hkv=1, d=2, page=16, q_len=q, kv_len=kv, seed=pick(1 << 20))
        s.table[pick(3), 0] = -1
        tree = None if pick(2) else torch.rand(s.n, 12, generator=g) < 0.4
        prefix = None if pick(2) else [pick(50) - 5 for _ in range(3)]
        window, sink = pick(2) * (1 + pick(20)), pick(2) * pick(20)
        for b in range(3):
            assert torch.equal(S.sight(s, b, prefix, window, sink, tree), K.sight(s, b, prefix, window, sink, tree))


def test_cuts_by_hand():
    """One request whose 64 new tokens are 512 rows of 8 heads' groups: 4 blocks, 32 groups."""
    one = cut([64], [300], 8, 1, 128, 16)
    assert one.blocks and not one.few and not one.groups and one.piece == 256 and one.pieces == 2 and one.join == 1
    assert one.workgroups == 1 + 2 + 2 + 2             # (the first block's tokens see 252 rows, the second's 268)
    few = cut([1, 2], [300, 40], 8, 1, 128, 16)
    assert few.few and not few.blocks and few.step_piece == 128 and few.step_pieces == 3 and few.workgroups == 0
    grouped = cut([64], [300], 8, 1, 128, 8)           # (one request's groups: 32, and one for a sequence's rest)
    assert grouped.groups == 33 and not grouped.blocks
    both = cut([64, 1], [300, 40], 8, 1, 128, 16)
    assert both.blocks and both.few
    # under a window of 100 of 5000 rows the longest has 16 slots of its page, 100, and 15 of other blocks' tokens
    assert cut([1], [5000], 8, 1, 128, 16, window=100, sink=4).step_pieces == 1 and cut([1], [5000], 8, 1, 128, 16).step_pieces > 8


def test_refusals_of_the_hook():
    for bad in [dict(bits=5), dict(d=32), dict(hq=7), dict(hq=34), dict(window=-1), dict(max_kv=-1), dict(cap=-1.0)]:
        kw = dict(q=[3], kv=[30], hq=8, hkv=2, d=64, bits=8)
        kw.update(bad)
        with pytest.raises(A.ArkvError):
            cut(**kw)
    assert P.load().arkv_debug_attention_cut(None, None, None, None, 8, None) == A.EINVAL
    with pytest.raises(A.ArkvError) as e:               # 2^27 workgroups
        cut([1] * (1 << 14), [5] * (1 << 14), 16, 16, 128, 8, max_kv=1 << 20)
    assert e.value.code == A.EUNSUPPORTED
    with pytest.raises(ValueError):
        P.arkv_debug_attention_cut([0, 1], [3, 4], 1, 1, 4, 8, 2, 64, 8)


@pytest.mark.parametrize("d,bits,cap,places", [(128, 8, 0.0, 512), (128, 4, 0.0, 512), (128, 16, 30.0, 512), (64, 16, 0.0, 768), (64, 8, 0.0, 768), (64, 8, 30.0, 768),
                                               (64, 4, 30.0, 768), (64, 4, 300.0, 768), (64, 4, 0.0, 512)])
def test_pieces_are_planned_for_the_places_of_the_build_that_runs(d, bits, cap, places):
    """Workgroups of four waves: three or two to each of 256 CUs, by the registers that the build leaves a wave."""
    window = 3000 if bits == 16 else 0
    c = cut([700, 700, 300], [5000, 4000, 6000], 16, 4, d, bits, window=window, cap=cap)
    assert c.blocks and c.pieces > 1 and c.places == places and c.workgroups <= places


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64), (16, 1, 64), (21, 3, 64), (4, 4, 64)])
def test_a_workspace_of_4_bit_pages_serves_every_window_and_cap(hq, hkv, d):
    """Their builds have other places than those of 8 bits, and others with a cap: no call may need more than the workspace's size."""
    if torch.cuda.is_available():
        pytest.skip("would launch")                    # (without a GPU a call that passes its checks fails in the launch)
    rng = np.random.default_rng(hq + d)
    lib, n, r, at = P.load(), C.c_size_t(), C.byref, 0x1000
    pages, rows = P._Packed(0, 4, 100, 64, hkv, d, at, at, at, at, at), P._Rows(at, hq * d, d)
    for _ in range(1500):
        batch, n_tokens, max_kv, window = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (500, 30000, 1 << 20, 1 << 20))
        max_q = min(n_tokens, int(np.exp(rng.uniform(0, np.log(n_tokens + 1)))))
        b = P._Batch(batch, n_tokens, max_q, max_kv, 1 << 20, at, at, at)
        assert lib.arkv_packed_workspace(r(pages), r(b), hq, r(n)) == A.OK
        for cap in (0.0, 30.0):
            for s in (None, P._Sight(window, 4, 0, None), P._Sight(window, 0, 1 << 10, at)):
                args = (r(pages), r(b), r(P._Scores(0.125, cap, None, None, None)), s if s is None else r(s), hq, r(rows), at, None, at)
                assert lib.arkv_packed_attention(*args, 0, None) == A.EINVAL
                assert lib.arkv_packed_attention(*args, n.value, None) in (A.EHIP, A.EUNSUPPORTED), (batch, n_tokens, max_q, max_kv, window, cap)


@pytest.mark.parametrize("q,kv,hq,hkv,d,bits,window", [
    ([3, 46, 1, 40, 494, 14, 1917], [3514, 6832, 157, 3426, 7817, 1857, 4591], 24, 8, 128, 8, 1990), ([3, 10, 2478], [1875, 6397, 4064], 32, 8, 64, 8, 536),
    ([2196, 60, 101, 181], [9849, 3010, 7089, 1188], 24, 8, 64, 4, 1413), ([129] * 40, [5000] * 40, 4, 4, 128, 16, 1600)])
def test_a_short_last_block_does_not_decide_for_those_before_it(q, kv, hq, hkv, d, bits, window):
    """Under a window a sequence's last block, of few tokens, has fewer keys than the others: they do not become two pieces each beyond the places."""
    c = cut(q, kv, hq, hkv, d, bits, window=window, sink=4)
    assert c.places and c.workgroups <= c.places


def test_pieces_fit_the_places_wherever_whole_blocks_do():
    rng, chosen = np.random.default_rng(5), 0
    for _ in range(6000):
        B, hkv, G = int(rng.integers(1, 9)), int(rng.choice([1, 2, 4, 8])), int(rng.choice([1, 2, 3, 4, 7, 8]))
        q = [int(np.exp(rng.uniform(0, np.log(2500)))) for _ in range(B)]
        kv = [a + int(rng.integers(0, 8000)) for a in q]
        window = int(rng.integers(0, 2)) * int(np.exp(rng.uniform(3, 8)))
        c = cut(q, kv, hkv * G, hkv, int(rng.choice([64, 128])), int(rng.choice([16, 8, 4])), window=window, sink=int(rng.integers(0, 70)), tree=bool(rng.integers(0, 2)))
        if c.places and sum(-(-a * G // 128) * hkv for a in q if a * G > 16) <= c.places:
            chosen += 1
            assert c.workgroups <= c.places, (q, kv, hkv, G, window, vars(c))
    assert chosen > 500
