"""Drafted tokens over packed pages: `python -m paper_2603_08727_amd.paged_drafts_example`.

One attention layer with random weights stands in for a model whose layers look `window` rows back and at a few first ones.
Requests keep their rows in 8 or 4 bits.  A round carries a tree of drafted tokens of every request: arkv_packed_append puts
them behind the accepted rows, arkv_packed_attention lets each see its ancestors; of the tree one path is accepted, whose rows
are appended again in the drafts' place.
"""
from __future__ import annotations

import math

import torch

from . import paged as P


class DraftedLayer:
    """One layer's packed pages and the requests in them, each with room for `rows` rows."""

    def __init__(self, n_requests, hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=64, bits=8, page_size=16, rows=1024, window=256, sink=4,
                 max_tokens=128, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.hq, self.hkv, self.d, self.rows, self.max_tokens, self.device = n_q_heads, n_kv_heads, head_dim, rows, max_tokens, device
        self.window, self.sink, self.scale = window, sink, 1.0 / math.sqrt(head_dim)
        width = -(-rows // page_size)
        pool = (n_requests * width, n_kv_heads, page_size)
        u8 = dict(dtype=torch.uint8, device=device)
        self.pages = P.arkv_packed_pages(torch.zeros(*pool, head_dim * bits // 8, **u8), torch.zeros(*pool, head_dim * bits // 8, **u8),
                                         torch.zeros(*pool, head_dim // 32, **u8), torch.zeros(*pool, head_dim // 32, **u8),
                                         torch.zeros(pool, dtype=torch.int32, device=device), dtype)
        self.w_qkv = (torch.randn(hidden, (n_q_heads + 2 * n_kv_heads) * head_dim, generator=g, device=device) / math.sqrt(hidden)).to(dtype)
        self.w_out = (torch.randn(n_q_heads * head_dim, hidden, generator=g, device=device) / math.sqrt(n_q_heads * head_dim)).to(dtype)
        half = head_dim // 2
        self.rotary = P.arkv_rotary(10000.0 ** (-torch.arange(half, dtype=torch.float64, device=device) / half))
        self.table = torch.randperm(n_requests * width, generator=g, device=device).to(torch.int32).reshape(n_requests, width)
        self.have = [0] * n_requests                   # accepted rows
        self.drafted = None                            # the round's keys, values and trees, until some of them are accepted
        lengths = torch.zeros(n_requests + 1, dtype=torch.int32, device=device)
        largest = P.arkv_page_batch(lengths, lengths[1:], self.table, n_requests * max_tokens, max_tokens, rows)
        self.workspace = P.arkv_packed_workspace(self.pages, largest, n_q_heads)       # serves every smaller batch

    def _batch(self, q_len):
        lens = [h + a for h, a in zip(self.have, q_len)]
        if max(q_len) > self.max_tokens or max(lens) > self.rows:
            raise ValueError(f"{q_len} tokens behind {self.have} rows: up to {self.max_tokens} tokens, {self.rows} rows")
        cu = torch.tensor([sum(q_len[:i]) for i in range(len(q_len) + 1)], dtype=torch.int32, device=self.device)
        return P.arkv_page_batch(cu, torch.tensor(lens, dtype=torch.int32, device=self.device), self.table, sum(q_len), max(q_len), max(lens))

    def _step(self, x, q_len, positions, tree):
        n, hq, hkv, d = x.shape[0], self.hq, self.hkv, self.d
        batch = self._batch(q_len)
        qkv = (x @ self.w_qkv).view(n, hq + 2 * hkv, d)
        k, v = qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        positions = torch.tensor([positions], dtype=torch.int32, device=self.device)
        q, out = (torch.empty(n, hq, d, dtype=x.dtype, device=self.device) for _ in range(2))
        P.arkv_packed_append(self.pages, batch, self.rotary, qkv[:, :hq], k, v, positions, q)
        P.arkv_packed_attention(self.pages, batch, q, self.scale, out, sight=P.arkv_sight(self.window, self.sink, tree), workspace=self.workspace)
        return out.reshape(n, hq * d) @ self.w_out, k, v

    def prompt(self, x, q_len):
        """x [sum(q_len)][hidden], request after request: accepted tokens, each of which sees those before it."""
        y, _, _ = self._step(x, q_len, [h + i for h, a in zip(self.have, q_len) for i in range(a)], None)
        self.drafted = None                            # (of a round that nothing was accepted of: the prompt's rows are in its place)
        self.have = [h + a for h, a in zip(self.have, q_len)]
        return y

    def draft(self, x, parents):
        """A tree of drafted tokens of every request: parents[r][i] is the draft that draft i follows, -1 the accepted rows.  The layer's
        output for each; nothing is accepted yet.  A window counts from a draft's place but takes no drafts away: trees are less deep than it."""
        q_len, depth, bits = [len(p) for p in parents], [], []
        words = max(1, -(-max(q_len) // 64))
        for p in parents:
            seen, at = [], []
            for i, up in enumerate(p):
                if not -1 <= up < i:
                    raise ValueError(f"draft {i} follows {up}: one before it, or -1")
                seen.append((seen[up] if up >= 0 else 0) | 1 << i)
                at.append(at[up] + 1 if up >= 0 else 0)
                if 0 < self.window <= at[i]:
                    raise ValueError(f"draft {i} follows {at[i]} others: its window of {self.window} would end within them")
            depth.append(at)
            bits += [[w - (1 << 64) if w >> 63 else w for w in (s >> 64 * j & (1 << 64) - 1 for j in range(words))] for s in seen]
        tree = torch.tensor(bits, dtype=torch.int64, device=self.device).reshape(-1, words)
        y, k, v = self._step(x, q_len, [h + i for h, at in zip(self.have, depth) for i in at], tree)
        self.drafted = (k, v, [list(p) for p in parents])
        return y

    def accept(self, paths):
        """The drafts of every request that are accepted, from the accepted rows on, each following the one before it: their rows take
        the drafts' place."""
        if self.drafted is None:
            raise ValueError("nothing is drafted")
        k, v, parents = self.drafted
        if len(paths) != len(parents):
            raise ValueError(f"{len(paths)} paths for {len(parents)} requests")
        for path, p in zip(paths, parents):
            for at, i in zip([-1, *path], path):
                if not 0 <= i < len(p) or p[i] != at:
                    raise ValueError(f"path {path}: draft {i} does not follow {at}")
        self.drafted, q_len = None, [len(p) for p in parents]
        picked = torch.tensor([sum(q_len[:r]) + i for r, path in enumerate(paths) for i in path], dtype=torch.int64, device=self.device)
        counts = [len(p) for p in paths]
        positions = torch.tensor([[h + i for h, a in zip(self.have, counts) for i in range(a)]], dtype=torch.int32, device=self.device)
        if sum(counts):
            P.arkv_packed_append(self.pages, self._batch(counts), self.rotary, None, k[picked], v[picked], positions, None)
        self.have = [h + a for h, a in zip(self.have, counts)]


def main():
    g = torch.Generator().manual_seed(0)
    layer = DraftedLayer(3, bits=8)
    y = layer.prompt(torch.randn(100 + 30 + 128, 512, generator=g).to(torch.bfloat16).cuda(), [100, 30, 128])
    print(f"prompts: rows {layer.have}, output {float(y.float().abs().mean()):.4f}", flush=True)
    for turn in range(8):
        parents = [[-1, 0, 0, 1, 1, 2, 3], [-1, 0, 1, 2], [-1, -1, 0, 1, 2, 2]]
        y = layer.draft(torch.randn(sum(map(len, parents)), 512, generator=g).to(torch.bfloat16).cuda(), parents)
        paths = []
        for p in parents:                              # (a model would take the drafts that its own choices agree with)
            path, at = [], -1
            while True:
                after = [i for i, up in enumerate(p) if up == at]
                if not after or torch.rand(1, generator=g) < 0.3:
                    break
                at = after[int(torch.randint(len(after), (1,), generator=g))]
                path.append(at)
            paths.append(path)
        layer.accept(paths)
        print(f"round {turn}: accepted {paths}, rows {layer.have}, output {float(y.float().abs().mean()):.4f}", flush=True)


if __name__ == "__main__":
    main()
