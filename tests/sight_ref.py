"""Which slots tokens see, as whole matrices (packed_ref.sight goes through them one by one), and attention by them: for sequences of many
tokens and rows.  And how a call over them is divided."""
from unittest import mock

import torch

from paper_2603_08727_amd import paged as P
import paged_ref as R


def sight(s, b, prefix=None, window=0, sink=0, tree=None):
    """[q][t], as packed_ref.sight."""
    t, a, at, dev = s.kv_len_list[b], s.q_len[b], sum(s.q_len[:b]), s.table.device
    ctx = t - a
    if not a:
        return torch.zeros(0, t, dtype=torch.bool, device=dev)
    i, j = torch.arange(a, device=dev)[:, None], torch.arange(t, device=dev)[None]
    if tree is None:
        place, see = ctx + i, j <= ctx + i
    else:
        mine = tree[at:at + a, :a].to(dev)
        place, see = ctx + (mine.sum(1, keepdim=True) - 1).clamp(min=0), (j < ctx).expand(a, t)
    if window:
        see = see & ((j > place - window) | (j < sink))
    if tree is not None:
        new = j[0] - ctx
        see = see | mine[:, new.clamp(min=0, max=a - 1)] & (new >= 0)[None]
    see = see & (ctx + i >= 0)
    if prefix is not None:
        see = see | (j < int(prefix[b]))
    return see & R.rows(s, s.pos, b, 0)[1][None]


def attention(s, window=0, sink=0, tree=None, **kw):
    """paged_ref.attention, every sequence's matrix made once."""
    made = {}

    def visible(s, b, prefix=None):
        if b not in made:
            made[b] = sight(s, b, prefix, window, sink, tree)
        return made[b]

    with mock.patch.object(R, "visible", visible):
        return R.attention(s, **kw)


class Cut:
    def __init__(self, numbers):
        (self.kinds, self.groups, self.step_piece, self.step_pieces, self.piece, self.pieces, self.join, self.workgroups, self.places) = numbers
        self.blocks, self.few = bool(self.kinds & 1), bool(self.kinds & 2)


def cut(s, window=0, sink=0, tree=None, cap=0.0, prefix=None, max_q=None, max_kv=None, **_):
    """How the call is divided: by blocks of 128 rows, groups of 16; pieces of a block, and what joins them."""
    max_q = s.max_q if max_q is None else max_q
    return Cut(P.arkv_debug_attention_cut(s.cu_q.cpu().numpy(), s.kv_len.cpu().numpy(), s.n, max_q, s.max_kv if max_kv is None else max_kv, s.hq, s.hkv, s.d,
                                          getattr(s, "bits", 16), window, sink, 0 if tree is None else max(1, -(-max_q // 64)), cap,
                                          None if prefix is None else prefix.cpu().numpy()))
