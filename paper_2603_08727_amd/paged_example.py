"""A small server on the paged operators: `python -m paper_2603_08727_amd.paged_example`.

One attention layer with random weights stands in for a model.  Requests of different lengths share a pool of pages; every
step carries a prompt chunk of one request beside a generated token of each of the others.  Per step and layer:
arkv_paged_append (rotary positions, rows into pages), arkv_paged_attention, arkv_paged_weights; a request whose rows
exceed the limit is cut to its budget by arkv_paged_evict into fresh pages, and its old pages return to the pool.
"""
from __future__ import annotations

import math

import torch

from . import paged as P


class PagedLayer:
    """One layer's pages, the requests in them, and the host's page bookkeeping."""

    def __init__(self, n_requests, hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=256, limit=256,
                 budget=128, max_tokens=256, dtype=torch.bfloat16, seed=0, device="cuda"):
        if not 0 < budget <= limit:
            raise ValueError(f"budget {budget}: a request over the limit of {limit} rows is cut to 1 .. limit of them")
        g = torch.Generator(device=device).manual_seed(seed)
        self.max_tokens = max_tokens                   # of a request in one step
        self.hq, self.hkv, self.d, self.page, self.limit, self.budget, self.device = n_q_heads, n_kv_heads, head_dim, page_size, limit, budget, device
        # a chunk can bring a request over its limit before it is cut
        self.width = -(-(limit + max_tokens) // page_size)
        self.w_qkv = (torch.randn(hidden, (n_q_heads + 2 * n_kv_heads) * head_dim, generator=g, device=device) / math.sqrt(hidden)).to(dtype)
        self.w_out = (torch.randn(n_q_heads * head_dim, hidden, generator=g, device=device) / math.sqrt(n_q_heads * head_dim)).to(dtype)
        pool = (n_pages, n_kv_heads, page_size)
        self.pages = P.arkv_pages(torch.zeros(*pool, head_dim, dtype=dtype, device=device), torch.zeros(*pool, head_dim, dtype=dtype, device=device),
                                  torch.zeros(pool, dtype=torch.int32, device=device), torch.zeros(pool, device=device))
        half = head_dim // 2
        self.rotary = P.arkv_rotary(10000.0 ** (-torch.arange(half, dtype=torch.float64, device=device) / half))
        self.free = list(range(n_pages))
        self.held = [[] for _ in range(n_requests)]    # pages of every request
        self.rows = [0] * n_requests                   # rows it has in them
        self.seen = [0] * n_requests                   # tokens it has had: the next one's position
        # the step's arrays live as long as the server: a captured step would find them where they were
        self.table = torch.full((n_requests, self.width), -1, dtype=torch.int32, device=device)
        lengths = torch.zeros(n_requests + 1, dtype=torch.int32, device=device)
        largest = P.arkv_page_batch(lengths, lengths[1:], self.table, n_requests * max_tokens, max_tokens, self.width * page_size)
        self.workspace = P.arkv_paged_workspace(self.pages, largest, n_q_heads)        # serves every smaller batch

    def _take(self, n):
        got, self.free = self.free[:n], self.free[n:]
        return got

    def _batch(self, q_len):
        dev = self.device
        for r, held in enumerate(self.held):
            if held:
                self.table[r, :len(held)] = torch.tensor(held, dtype=torch.int32, device=dev)
        cu = torch.tensor([sum(q_len[:i]) for i in range(len(q_len) + 1)], dtype=torch.int32, device=dev)
        return P.arkv_page_batch(cu, torch.tensor(self.rows, dtype=torch.int32, device=dev), self.table, sum(q_len), max(q_len),
                                 max(self.rows))

    def _check_step(self, n, q_len):
        if len(q_len) != len(self.rows) or sum(q_len) != n or not all(0 <= a <= self.max_tokens for a in q_len):
            raise ValueError(f"{n} tokens as {q_len}: one count of 0 to {self.max_tokens} for each of {len(self.rows)} requests")
        rows = [have + a for have, a in zip(self.rows, q_len)]
        need = sum(-(-m // self.page) - len(held) for m, held in zip(rows, self.held))
        need += sum(m > self.limit for m in rows) * -(-self.budget // self.page)       # (the old pages return behind the eviction)
        if need > len(self.free):
            raise RuntimeError(f"out of pages: {need} wanted, {len(self.free)} free")

    def step(self, x, q_len):
        """x [sum(q_len)][hidden], request after request: the layer's output for the new tokens.  A step that is refused (too many
        tokens, not enough pages) changes nothing."""
        n, hq, hkv, d = x.shape[0], self.hq, self.hkv, self.d
        self._check_step(n, q_len)
        qkv = (x @ self.w_qkv).view(n, hq + 2 * hkv, d)
        positions = []
        for r, a in enumerate(q_len):
            positions += range(self.seen[r], self.seen[r] + a)
            self.seen[r] += a
            self.rows[r] += a
            self.held[r] += self._take(-(-self.rows[r] // self.page) - len(self.held[r]))
        batch = self._batch(q_len)
        positions = torch.tensor([positions], dtype=torch.int32, device=self.device)
        q, out, lse = (torch.empty(n, hq, d, dtype=x.dtype, device=self.device), torch.empty(n, hq, d, dtype=x.dtype, device=self.device),
                       torch.empty(n, hq, device=self.device))
        scale = 1.0 / math.sqrt(d)
        P.arkv_paged_append(self.pages, batch, self.rotary, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], positions, q)
        P.arkv_paged_attention(self.pages, batch, q, scale, out, lse=lse, workspace=self.workspace)
        P.arkv_paged_weights(self.pages, batch, q, scale, lse, workspace=self.workspace)
        self._evict(batch)
        return out.reshape(n, hq * d) @ self.w_out

    def _evict(self, batch):
        """Cuts the requests over the limit to the budget; the others keep no row in the call and stay where they are."""
        over = [r for r, n in enumerate(self.rows) if n > self.limit]
        if not over:
            return
        need = -(-self.budget // self.page)
        keep = torch.zeros(len(self.rows), dtype=torch.int32, device=self.device)
        dst = torch.full((len(self.rows), need), -1, dtype=torch.int32, device=self.device)
        fresh = {}
        for r in over:
            fresh[r] = self._take(need)
            keep[r] = self.budget
            dst[r] = torch.tensor(fresh[r], dtype=torch.int32, device=self.device)
        kept = torch.empty((len(self.rows), self.hkv, self.budget), dtype=torch.int32, device=self.device)
        new_len = torch.empty(len(self.rows), dtype=torch.int32, device=self.device)
        P.arkv_paged_evict(self.pages, batch, keep, dst, kept, new_len, sink=4, recent=32, workspace=self.workspace)
        for r in over:
            self.free += self.held[r]                  # (the next writes into them come behind this call on the same stream)
            self.held[r], self.rows[r] = fresh[r], self.budget


def main():
    torch.manual_seed(0)
    prompts, chunk, steps = [700, 90, 333, 20], 128, 40
    layer = PagedLayer(len(prompts), max_tokens=chunk)
    todo, x_of = list(prompts), {}
    for step in range(steps):
        # one prompt chunk at a time; requests whose prompt is through generate
        first = next((r for r, n in enumerate(todo) if n), None)
        q_len = [0] * len(prompts)
        for r, n in enumerate(todo):
            if r == first:
                q_len[r] = min(chunk, n)
                todo[r] -= q_len[r]
            elif not n and layer.seen[r]:
                q_len[r] = 1
        x = torch.randn(sum(q_len), 512, device="cuda").to(torch.bfloat16)
        y = layer.step(x, q_len)
        if step % 8 == 0 or step == steps - 1:
            print(f"step {step:3d}: new tokens {q_len}, rows {layer.rows}, seen {layer.seen}, free pages {len(layer.free)}, "
                  f"output {float(y.float().abs().mean()):.4f}", flush=True)


if __name__ == "__main__":
    main()
