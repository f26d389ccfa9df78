"""Timed cases of the operators around a paged cache: rotary positions on the way into the pages, attention of new
tokens over them, the attention weight that their rows collected, eviction by that weight.

`listed()` is the fixed list, `draw()` gives further cases of the same ranges, `prepare()` makes what a serving program
has in hand before a call, `run()` is one pass through an operator (`own`: through paper_2603_08727_amd.paged, else the
plain form in elementary torch operations), `work()` says what a pass cannot do without, `exact()` is the result in 64
bits, one sequence at a time.

A sequence's rows lie in pages of `page` slots: `table[b][j // page]` is the page of its slot j, and a page holds its
rows for every kv-head, [page][kv-head][slot][channel].  `kv_len[b]` counts the sequence's rows, its `q_len[b]` new
tokens (the last ones) among them; the new tokens of all sequences lie one after the other, `cu_q` says where.

Kinds:
  append   rotary positions (one axis, or three) on q and k of the new tokens; k, v, position into the pages
  attend   softmax(q k^T) v of the new tokens over the pages: causal by slot, optionally with a capped score, a bias
           by distance, a prefix that every new token sees
  weigh    what those tokens' probabilities add to the weight of every cached row
  evict    every kv-head's rows of least weight leave: survivors go to fresh pages, in order
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, kind, **kw):
    c = dict(kind=kind, dtype="bf16", hq=32, hkv=8, d=128, page=16, batch=1, q="one", q_max=1, kv_max=1024, spread=0.0,
             idle=False, lens=0, cap=0.0, distance=False, prefix=False, axes=1, rot=0, adjacent=False, decay=1.0,
             keep=0, sink=4, recent=32)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one generated token of each of sixteen requests on its way into the cache: a launch's latency
        _case("append_step", "append", batch=16, kv_max=2048, spread=0.5, rot=128),
        # prompt chunks of an image-text model: positions along time, height and width, ragged chunks
        _case("append_image_chunks", "append", batch=4, q="ragged", q_max=2731, kv_max=9000, spread=0.6, axes=3, rot=128),
        # the smallest call: one token of one request of a small model
        _case("attend_step_small", "attend", dtype="fp16", hq=8, hkv=2, d=64, kv_max=513),
        # a step of a busy server: many requests of very different lengths, one slot of the batch idle
        _case("attend_step_ragged", "attend", batch=32, kv_max=16384, spread=0.95, idle=True),
        # four requests of 128K tokens, 64 query heads on 8 kv-heads
        _case("attend_step_128k", "attend", hq=64, batch=4, kv_max=131071, page=64),
        # a step that carries one prompt chunk beside single tokens of others; capped scores, a kv-head per query head
        _case("attend_mixed_capped", "attend", hq=16, hkv=16, batch=8, q="mixed", q_max=512, kv_max=4100, spread=0.7, cap=30.0),
        # a chunk of two long prompts
        _case("attend_chunk_16k", "attend", batch=2, q="all", q_max=2048, kv_max=16384, page=64),
        # odd chunks behind an image prefix that sees itself whole; bias by distance; three query heads per kv-head
        _case("attend_prefix_distance", "attend", dtype="fp16", hq=12, hkv=4, d=64, batch=3, q="ragged", q_max=777,
              kv_max=3001, spread=0.5, distance=True, prefix=True),
        # what one step's tokens looked at, weights fading from step to step
        _case("weigh_step", "weigh", batch=16, kv_max=8192, spread=0.3, decay=0.9375),
        # what a prompt's last chunk looked at
        _case("weigh_chunk", "weigh", batch=2, q="all", q_max=1024, kv_max=8191),
        # short requests over their budget
        _case("evict_small", "evict", hq=8, hkv=2, d=64, batch=8, kv_max=1000, spread=0.4, keep=250),
        # prompts of 32K tokens on their way to a quarter
        _case("evict_32k", "evict", batch=4, kv_max=32768, page=64, keep=8192),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "weigh", "evict"])
    hkv, g = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 3, 4, 8])
    while hkv * g > 64:
        g = rng.choice([1, 2, 3, 4])
    d = rng.choice([64, 128])
    kw = dict(dtype=rng.choice(["bf16", "fp16"]), hkv=hkv, hq=hkv * g, d=d, page=rng.choice([16, 16, 32, 64, 128]),
              batch=_log(rng, 1, 32), spread=rng.choice([0.0, 0.3, 0.6, 0.95]), lens=rng.randrange(1 << 30))
    rows = 4 * 131072 * 8 * 128 // (hkv * d)                # of all sequences: what the largest listed cache holds
    if kind == "append":
        q = rng.choice(["one", "ragged", "mixed", "all"])
        q_max = 1 if q == "one" else _log(rng, 2, min(4096, 8192 * 48 // ((hkv * g + 2 * hkv) * kw["batch"])) )
        axes = rng.choice([1, 2, 3])
        return _case(None, kind, q=q, q_max=q_max, kv_max=q_max + _log(rng, 1, 8192), axes=axes,
                     rot=rng.choice([d, d, d // 2]), adjacent=rng.random() < 0.3, **kw)
    if kind == "evict":
        kv_max = _log(rng, 40, max(41, min(65536, 4 * 32768 * 8 * 128 // (hkv * d * kw["batch"]))))
        return _case(None, kind, kv_max=kv_max, keep=max(36, int(kv_max * rng.choice([0.125, 0.25, 0.5, 0.8]))), **kw)
    q = rng.choice(["one", "one", "mixed", "ragged", "all"])
    if q == "one":
        kv_max = _log(rng, 16, min(131072, max(17, rows // (2 * kw["batch"]))))
        q_max = 1
    else:
        pairs = 2 * 2048 * 16384 * 32 // (2 * hkv * g * kw["batch"])     # half the largest listed case's scores
        q_max = _log(rng, 2, min(2048, max(3, pairs // 64)))
        kv_max = q_max + _log(rng, 1, max(2, min(16384, pairs // q_max)))
    more = {}
    if kind == "weigh":
        more["decay"] = rng.choice([0.0, 0.5, 0.9375, 1.0])
    else:
        more = rng.choice([{}, {}, {"cap": rng.choice([20.0, 30.0, 50.0])}, {"distance": True}, {"prefix": q != "one"}])
    return _case(None, kind, q=q, q_max=q_max, kv_max=kv_max, idle=kw["batch"] > 2 and rng.random() < 0.3, **more, **kw)


def _lengths(c):
    """(q_len, kv_len) of every sequence, from the case alone."""
    r = random.Random(c["lens"])
    q, kv = [], []
    for b in range(c["batch"]):
        f = 1.0 if b == 0 else 1.0 - c["spread"] * r.random()
        if c["q"] in ("one", "all"):
            n = c["q_max"]
        elif c["q"] == "mixed":
            n = c["q_max"] if b == 0 else 1
        else:
            n = max(1, int(c["q_max"] * (1.0 if b == 0 else 1.0 - 0.8 * r.random())))
        if c["idle"] and b == c["batch"] - 1:
            n, t = 0, 0
        else:
            t = max(n, int(c["kv_max"] * f))
        q.append(n)
        kv.append(t)
    return q, kv


def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 17)
    dt = DTYPES[c["dtype"]]
    B, hq, hkv, d, ps = c["batch"], c["hq"], c["hkv"], c["d"], c["page"]
    q_len, kv_len = _lengths(c)
    need = [-(-t // ps) for t in kv_len]
    keep_pages = -(-c["keep"] // ps)
    n_pages = sum(need) + B * keep_pages + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    width = max(need) + 1
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    s = dict(case=c, n=sum(q_len), max_q=max(q_len), max_kv=max(kv_len), table=table)
    s["cu_q"] = torch.tensor([sum(q_len[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
    s["kv_len"] = torch.tensor(kv_len, dtype=torch.int32, device=dev)
    n = s["n"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    # rows that a model's cache holds: two channels stand out, the first rows of a sequence draw attention
    lift = torch.ones(d, device=dev)
    lift[[3, d // 2 + 3]] = 4.0
    k = normal(n_pages, hkv, ps, d) * lift
    first = table[:, 0][table[:, 0] >= 0].long()
    k[first, :, :4] *= 2.0
    s["k"] = k.to(dt)
    del k
    s["v"] = normal(n_pages, hkv, ps, d).to(dt)
    s["pos"] = torch.full((n_pages, hkv, ps), -1, dtype=torch.int32, device=dev)
    s["weight"] = torch.zeros((n_pages, hkv, ps), device=dev)
    ctx = (s["kv_len"] - (s["cu_q"][1:] - s["cu_q"][:-1])).tolist()
    shift = [int(x) for x in torch.randint(0, 1000, (B,), generator=g, device=dev)]   # rows that left before
    if c["kind"] in ("attend", "weigh"):
        # heads differ in how sharply they look
        temp = torch.where(torch.rand(hq, generator=g, device=dev) < 0.5, 0.6, 1.8)
        fused = torch.empty((n, hq + 2 * hkv, d), dtype=dt, device=dev)               # a fused projection's output
        fused[:] = normal(n, hq + 2 * hkv, d).to(dt)
        fused[:, :hq] = (fused[:, :hq].float() * temp[None, :, None]).to(dt)
        s["q"] = fused[:, :hq]
        s["scale"] = 1.0 / math.sqrt(d)
        slot = torch.arange(width * ps, device=dev, dtype=torch.int32)
        for b in range(B):
            p = (slot + shift[b] * (slot >= 4)).int()
            s["pos"][table[b, :need[b]].long()] = p.reshape(width, 1, ps)[:need[b]].expand(-1, hkv, -1)
        s["q_pos"] = torch.cat([torch.arange(ctx[b], ctx[b] + q_len[b], device=dev, dtype=torch.int32) +
                                (shift[b] if ctx[b] >= 4 else 0) for b in range(B)])
        s["slopes"] = 2.0 ** (-8.0 * (torch.arange(hq, device=dev, dtype=torch.float32) + 1) / hq) if c["distance"] else None
        if c["prefix"]:
            s["prefix"] = torch.tensor([min(kv_len[b], ctx[b] + (2 * q_len[b]) // 3) for b in range(B)], dtype=torch.int32, device=dev)
        else:
            s["prefix"] = None
        s["out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
        s["lse"] = torch.empty((n, hq), dtype=torch.float32, device=dev)
    if c["kind"] == "weigh":
        s["carried"] = torch.rand((n_pages, hkv, ps), generator=g, device=dev)
        s["lse"] = _attend(s)["lse"]                                                   # the attention's, run before
    if c["kind"] == "append":
        fused = normal(n, hq + 2 * hkv, d).to(dt)
        s["q"], s["new_k"], s["new_v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        s["q_out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
        base = torch.cat([torch.arange(ctx[b], ctx[b] + q_len[b], device=dev, dtype=torch.int32) + 30 * shift[b] for b in range(B)])
        grid = [base, base % 27, base // 27 % 31]                                      # time, height, width
        s["positions"] = torch.stack(grid[:c["axes"]]).contiguous()
        half = c["rot"] // 2
        s["freq"] = 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        s["axis"] = [0] * half if c["axes"] == 1 else [min(c["axes"] - 1, i * c["axes"] // half) for i in range(half)]
        s["axis_dev"] = torch.tensor(s["axis"], device=dev)
    if c["kind"] == "evict":
        # few rows hold most of the weight; equal weights (rows nobody looked at) are common
        w = torch.rand((n_pages, hkv, ps), generator=g, device=dev)
        s["weight"] = torch.where(w < 0.25, torch.zeros_like(w), -torch.log(w) ** 3)
        s["weight"] = s["weight"].abs()
        s["pos"] = torch.randint(0, 1 << 20, (n_pages, hkv, ps), generator=g, device=dev, dtype=torch.int32)
        s["keep"] = torch.tensor([c["keep"]] * B, dtype=torch.int32, device=dev)
        s["dst_table"] = order[at:at + B * keep_pages].reshape(B, keep_pages).contiguous()
        s["kept"] = torch.empty((B, hkv, c["keep"]), dtype=torch.int32, device=dev)
        s["new_len"] = torch.empty(B, dtype=torch.int32, device=dev)
    if own:
        from paper_2603_08727_amd import paged as P
        s["pages"] = P.arkv_pages(s["k"], s["v"], s["pos"], s["weight"])
        s["batch"] = P.arkv_page_batch(s["cu_q"], s["kv_len"], s["table"], n, s["max_q"], s["max_kv"])
        s["workspace"] = P.arkv_paged_workspace(s["pages"], s["batch"], hq)
        if c["kind"] == "append":
            s["rotary"] = P.arkv_rotary(s["freq"], s["axis"], c["axes"], adjacent=c["adjacent"])
    return s


# ---- plain forms ------------------------------------------------------------------------------

def _tokens(s):
    """Sequence of every new token, and its index among that sequence's new ones."""
    t = torch.arange(s["n"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu_q"][1:].contiguous(), t, right=True)
    return b, t - s["cu_q"][b]


def _append(s):
    c = s["case"]
    hkv, d, ps, half = c["hkv"], c["d"], c["page"], c["rot"] // 2
    b, i = _tokens(s)
    angle = s["positions"][s["axis_dev"]].double() * s["freq"][:, None]                # [half][n]
    cos, sin = angle.cos().float().t()[:, None], angle.sin().float().t()[:, None]

    def turned(x):
        x = x.float()
        y = x.clone()
        if c["adjacent"]:
            a, e = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - e * sin, e * cos + a * sin
        else:
            a, e = x[..., :half], x[..., half:2 * half]
            y[..., :half], y[..., half:2 * half] = a * cos - e * sin, e * cos + a * sin
        return y.to(s["k"].dtype)

    slot = s["kv_len"][b] - (s["cu_q"][b + 1] - s["cu_q"][b]) + i
    page, off = s["table"][b, (slot // ps).long()].long(), (slot % ps).long()
    s["k"][page, :, off] = turned(s["new_k"])
    s["v"][page, :, off] = s["new_v"]
    s["pos"][page, :, off] = s["positions"][0][:, None].expand(-1, hkv)
    s["weight"][page, :, off] = 0.0
    return {"q": turned(s["q"]), "k": s["k"], "v": s["v"], "pos": s["pos"], "weight": s["weight"]}


def _dense(s, name):
    """[B][kv-head][slot][...] of a pool."""
    x = s[name][s["table"].clamp(min=0).long()]                                        # [B][pages][kv-head][slot]...
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])[:, :, :s["max_kv"]]


def _scores(s):
    """Scores [B][kv-head][head of the group][new token][slot], -inf where a token does not see the slot."""
    c = s["case"]
    B, hq, hkv, d, mq, mk = c["batch"], c["hq"], c["hkv"], c["d"], s["max_q"], s["max_kv"]
    q_len = s["cu_q"][1:] - s["cu_q"][:-1]
    i, j = torch.arange(mq, device="cuda"), torch.arange(mk, device="cuda")
    tok = (s["cu_q"][:-1, None] + i).clamp(max=s["n"] - 1)
    q = s["q"][tok].float().permute(0, 2, 1, 3).reshape(B, hkv, hq // hkv * mq, d)
    x = torch.matmul(q, _dense(s, "k").float().transpose(2, 3).contiguous()).mul_(s["scale"])
    x = x.reshape(B, hkv, hq // hkv, mq, mk)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if s["slopes"] is not None:
        far = (s["q_pos"][tok][:, None, :, None] - _dense(s, "pos")[:, :, None, :]).abs().float()
        x = x - s["slopes"].reshape(1, hkv, hq // hkv, 1, 1) * far[:, :, None]
    last = (s["kv_len"] - q_len)[:, None] + i
    if s["prefix"] is not None:
        last = torch.maximum(last, s["prefix"][:, None] - 1)
    seen = (j <= last[..., None]) & (j < s["kv_len"][:, None, None])
    return x.masked_fill_(~seen[:, None, None], -math.inf)


def _attend(s):
    c = s["case"]
    B, hq, hkv, d, mq = c["batch"], c["hq"], c["hkv"], c["d"], s["max_q"]
    x = _scores(s)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.reshape(B, hkv, -1, s["max_kv"]), _dense(s, "v").float().contiguous())
    out = out.reshape(B, hkv, hq // hkv, mq, d) / total
    lse = top + total.log()
    b, i = _tokens(s)
    out = out.reshape(B, hq, mq, d)[b, :, i.long()]
    return {"out": out.to(s["out"].dtype), "lse": lse.reshape(B, hq, mq)[b, :, i.long()]}


def _weigh(s):
    c = s["case"]
    B, hq, hkv, ps, mq, mk = c["batch"], c["hq"], c["hkv"], c["page"], s["max_q"], s["max_kv"]
    tok = (s["cu_q"][:-1, None] + torch.arange(mq, device="cuda")).clamp(max=s["n"] - 1)
    real = torch.arange(mq, device="cuda") < (s["cu_q"][1:] - s["cu_q"][:-1])[:, None]
    lse = s["lse"][tok].permute(0, 2, 1).masked_fill(~real[:, None], math.inf)
    p = _scores(s).sub_(lse.reshape(B, hkv, hq // hkv, mq, 1)).exp_()
    p = p.sum((2, 3))                                                                  # [B][kv-head][slot]
    j = torch.arange(mk, device="cuda")
    b, j = torch.nonzero(j < s["kv_len"][:, None], as_tuple=True)
    page, off = s["table"][b, j // ps].long(), j % ps
    s["weight"][page, :, off] = c["decay"] * s["carried"][page, :, off] + p[b, :, j]
    return {"weight": s["weight"]}


def _evict(s):
    c = s["case"]
    hkv, ps = c["hkv"], c["page"]
    n = s["kv_len"]
    m = torch.minimum(n, s["keep"])
    front = m.clamp(max=c["sink"])
    back = (m - front).clamp(max=c["recent"])
    j = torch.arange(s["max_kv"], device="cuda")
    w = _dense(s, "weight").nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    held = (j < front[:, None]) | ((j >= (n - back)[:, None]) & (j < n[:, None]))
    rank = torch.where(held, 2, torch.where(j < n[:, None], 1, 0))[:, None].expand(-1, hkv, -1)
    by_w = torch.sort(w, dim=-1, descending=True, stable=True).indices
    by_rank = torch.sort(rank.gather(2, by_w), dim=-1, descending=True, stable=True).indices
    order = by_w.gather(2, by_rank)                                                    # best first, ties to the lower slot
    width = min(c["keep"], s["max_kv"])
    slot = torch.arange(width, device="cuda")
    taken = torch.where(slot < m[:, None, None], order[..., :width], s["max_kv"]).sort(dim=-1).values
    real = slot < m[:, None, None].expand(-1, hkv, -1)
    kept = torch.full((c["batch"], hkv, c["keep"]), -1, dtype=torch.int32, device="cuda")
    kept[..., :width] = torch.where(real, taken, -1).int()
    b, h, to = torch.nonzero(real, as_tuple=True)
    src = taken[b, h, to]
    sp, so = s["table"][b, src // ps].long(), src % ps
    dp, do = s["dst_table"][b, to // ps].long(), to % ps
    for name in ("k", "v", "pos", "weight"):
        s[name][dp, h, do] = s[name][sp, h, so]
    return {"kept": kept, "new_len": m, "k": s["k"], "v": s["v"], "pos": s["pos"], "weight": s["weight"]}


def run(s):
    c = s["case"]
    if not own:
        return {"append": _append, "attend": _attend, "weigh": _weigh, "evict": _evict}[c["kind"]](s)
    from paper_2603_08727_amd import paged as P
    if c["kind"] == "append":
        P.arkv_paged_append(s["pages"], s["batch"], s["rotary"], s["q"], s["new_k"], s["new_v"], s["positions"], s["q_out"])
        return {"q": s["q_out"], "k": s["k"], "v": s["v"], "pos": s["pos"], "weight": s["weight"]}
    if c["kind"] == "attend":
        P.arkv_paged_attention(s["pages"], s["batch"], s["q"], s["scale"], s["out"], lse=s["lse"], cap=c["cap"],
                               slopes=s["slopes"], q_pos=s["q_pos"], prefix=s["prefix"], workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "weigh":
        P.arkv_paged_weights(s["pages"], s["batch"], s["q"], s["scale"], s["lse"], decay=c["decay"], carried=s["carried"],
                             cap=c["cap"], slopes=s["slopes"], q_pos=s["q_pos"], prefix=s["prefix"], workspace=s["workspace"])
        return {"weight": s["weight"]}
    P.arkv_paged_evict(s["pages"], s["batch"], s["keep"], s["dst_table"], s["kept"], s["new_len"], sink=c["sink"],
                       recent=c["recent"], workspace=s["workspace"])
    return {"kept": s["kept"], "new_len": s["new_len"], "k": s["k"], "v": s["v"], "pos": s["pos"], "weight": s["weight"]}


# ---- what a pass cannot do without ------------------------------------------------------------

def work(case):
    c = case
    q_len, kv_len = _lengths(c)
    n, rows = sum(q_len), sum(kv_len)
    d, hq, hkv, el = c["d"], c["hq"], c["hkv"], 2
    meta = 4 * (2 * c["batch"] + 1 + sum(-(-t // c["page"]) for t in kv_len))
    if c["kind"] == "append":
        fl = 3.0 * n * (hq + hkv) * c["rot"]
        return {"bytes": n * (2 * (hq + 2 * hkv) * d * el + 8 * hkv + 4 * c["axes"]) + meta, "flops": fl}
    if c["kind"] == "evict":
        m = sum(min(t, c["keep"]) for t in kv_len)
        return {"bytes": rows * hkv * 4 + m * hkv * (2 * (2 * d * el + 4) + 4 + 4) + meta, "flops": rows * hkv}
    pairs = 0
    for a, t in zip(q_len, kv_len):
        ctx = t - a
        p = ctx + (2 * a) // 3 if c["prefix"] else 0
        pairs += sum(max(ctx + i + 1, p) for i in range(a))
    if c["kind"] == "attend":
        return {"bytes": rows * hkv * (2 * d * el + (4 if c["distance"] else 0)) + n * hq * (2 * d * el + 4) + meta,
                "flops": 4.0 * d * pairs * hq}
    return {"bytes": rows * hkv * (d * el + 8) + n * hq * (d * el + 4) + meta, "flops": 2.0 * d * pairs * hq}


# ---- the same in 64 bits, one sequence at a time ------------------------------------------------

def _rows_of(s, name, b, t):
    """[kv-head][t][...] of a sequence's slots, in slot order."""
    ps = s["case"]["page"]
    pages = [int(x) for x in s["table"][b, :-(-t // ps)].tolist()]
    return torch.cat([s[name][p] for p in pages], dim=1)[:, :t]


def _exact_logits(s, b, h, q, k, q_len, kv_len, at):
    c = s["case"]
    x = (q.double() @ k.double().t()) * s["scale"]
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    t, a = kv_len[b], q_len[b]
    if s["slopes"] is not None:
        kp = _rows_of(s, "pos", b, t)[h // (c["hq"] // c["hkv"])].double()
        x = x - s["slopes"][h].double() * (s["q_pos"][at:at + a].double()[:, None] - kp[None, :]).abs()
    see = torch.arange(t, device="cuda")[None, :] <= (t - a + torch.arange(a, device="cuda"))[:, None]
    if s["prefix"] is not None:
        see = see | (torch.arange(t, device="cuda")[None, :] < int(s["prefix"][b]))
    return torch.where(see, x, torch.full_like(x, -math.inf))


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    q_len, kv_len = _lengths(c)
    n, hq, hkv, d, ps = s["n"], c["hq"], c["hkv"], c["d"], c["page"]
    grp = hq // hkv
    if c["kind"] == "append":
        half = c["rot"] // 2
        out = {"q": s["q"].double().clone(), "k": s["k"].double(), "v": s["v"].double(), "pos": s["pos"].clone(),
               "weight": s["weight"].double()}
        at = 0
        first, second = [], []
        for i in range(half):
            first.append(2 * i if c["adjacent"] else i)
            second.append(2 * i + 1 if c["adjacent"] else i + half)
        for b in range(c["batch"]):
            a = q_len[b]
            if not a:
                continue
            pos = s["positions"][:, at:at + a].double()
            turn = torch.polar(torch.ones(a, half, dtype=torch.float64, device="cuda"),
                               torch.stack([pos[ax] * s["freq"][i] for i, ax in enumerate(s["axis"])], dim=1))
            kk = s["new_k"][at:at + a].double().clone()
            for x in (out["q"][at:at + a], kk):
                z = torch.complex(x[..., first], x[..., second]) * turn[:, None, :]
                x[..., first], x[..., second] = z.real, z.imag
            slot = torch.arange(kv_len[b] - a, kv_len[b], device="cuda")
            page, off = s["table"][b][slot // ps].long(), slot % ps
            out["k"][page, :, off] = kk
            out["v"][page, :, off] = s["new_v"][at:at + a].double()
            out["pos"][page, :, off] = s["positions"][0, at:at + a, None].expand(-1, hkv)
            out["weight"][page, :, off] = 0.0
            at += a
        return out
    if c["kind"] == "evict":
        kept = torch.full((c["batch"], hkv, c["keep"]), -1, dtype=torch.int32)
        for b in range(c["batch"]):
            t = kv_len[b]
            m = min(t, c["keep"])
            f = min(c["sink"], m)
            r = min(c["recent"], m - f)
            w = _rows_of(s, "weight", b, t).double().cpu()
            middle = w[:, f:t - r]
            for h in range(hkv):
                best = torch.sort(middle[h], descending=True, stable=True).indices[:m - f - r] + f
                kept[b, h, :m] = torch.cat([torch.arange(f), torch.sort(best).values, torch.arange(t - r, t)]).int()
        out = {"kept": kept, "new_len": torch.tensor([min(t, c["keep"]) for t in kv_len], dtype=torch.int32)}
        for name in ("k", "v", "pos", "weight"):
            pool = s[name].clone() if name == "pos" else s[name].double()
            for b in range(c["batch"]):
                m = min(kv_len[b], c["keep"])
                rows = _rows_of(s, name, b, kv_len[b])
                to = torch.arange(m, device="cuda")
                page, off = s["dst_table"][b][to // ps].long(), to % ps
                for h in range(hkv):
                    pool[page, h, off] = rows[h, kept[b, h, :m].long().cuda()].to(pool.dtype)
            out[name] = pool
        return out
    out = torch.zeros((n, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((n, hq), dtype=torch.float64, device="cuda")
    weight = s["weight"].double()
    at = 0
    for b in range(c["batch"]):
        a, t = q_len[b], kv_len[b]
        if t:
            k, v = _rows_of(s, "k", b, t), _rows_of(s, "v", b, t)
            for g in range(hkv):
                total = torch.zeros(t, dtype=torch.float64, device="cuda")
                for h in range(g * grp, (g + 1) * grp):
                    x = _exact_logits(s, b, h, s["q"][at:at + a, h], k[g], q_len, kv_len, at)
                    if c["kind"] == "attend":
                        z = torch.logsumexp(x, dim=1)
                        out[at:at + a, h] = torch.exp(x - z[:, None]) @ v[g].double()
                        lse[at:at + a, h] = z
                    else:
                        total += torch.exp(x - s["lse"][at:at + a, h].double()[:, None]).sum(0)
                if c["kind"] == "weigh":
                    slot = torch.arange(t, device="cuda")
                    page, off = s["table"][b][slot // ps].long(), slot % ps
                    weight[page, g, off] = c["decay"] * s["carried"][page, g, off].double() + total
        at += a
    return {"out": out, "lse": lse} if c["kind"] == "attend" else {"weight": weight}
