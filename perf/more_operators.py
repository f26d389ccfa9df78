"""Timed cases of the paged cache's packed pages, and of attention that does not look at all rows before a token.

`listed()` is the fixed list, `draw()` gives further cases of the same ranges, `prepare()` makes what a serving program
has in hand before a call, `run()` is one pass (`own`: through paper_2603_08727_amd.paged, else the plain form in
elementary torch operations), `work()` says what a pass cannot do without, `exact()` is the result in 64 bits.

Pages, tables and lengths are those of perf/operators.py.  Packed pages hold a row of d channels in blocks of 32: a code
of 8 bits (sign, 4 of exponent with bias 7, 3 of mantissa) or 4 bits (1, 2 with bias 1, 1) per channel, the even channel
of a pair in a byte's low half, and a byte s per block; a channel is its code's value times 2^(s - 127).  s is the
smallest (from 1 on) for which the block's largest magnitude is at most 448 or 6 times that, the code the nearest one,
ties to the even one.

Kinds:
  store    rotary positions on q and k of the new tokens, their rows into packed pages; and the new rows read back
  fetch    whole sequences' rows out of packed pages, as a program takes them that goes on in 16 bits
  attend   softmax(q k^T) v of the new tokens over pages of 16, 8 or 4 bits.  A token at slot p sees the slots j <= p;
           window w > 0: of these j > p - w and j < sink; tree: a new token sees the rows before the new ones, and those
           new ones that its bits name (with a window, p is then the first new slot plus the number of tokens above it)
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FORMS = {8: (7, 3, 448.0), 4: (1, 1, 6.0)}            # bits: bias of the exponent, bits of the mantissa, largest value


def _case(name, kind, **kw):
    c = dict(kind=kind, dtype="bf16", bits=8, hq=32, hkv=8, d=128, page=16, batch=1, q="one", q_max=1, kv_max=1024, spread=0.0,
             idle=False, lens=0, window=0, sink=0, tree=False, cap=0.0, axes=1, rot=0, adjacent=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one generated token of each of sixteen requests on its way into an 8-bit cache: launches' latency
        _case("store_step_8", "store", batch=16, kv_max=2048, spread=0.5, rot=128),
        # ragged prompt chunks of an image-text model into a 4-bit cache
        _case("store_chunks_4", "store", bits=4, batch=4, q="ragged", q_max=2731, kv_max=9000, spread=0.6, axes=3, rot=128),
        # the first part of a conversation, back in 16 bits for one that branches off
        _case("fetch_short_4", "fetch", dtype="fp16", bits=4, hq=8, hkv=2, d=64, batch=3, q="whole", kv_max=777, spread=0.5),
        # long prompts out of an 8-bit cache
        _case("fetch_long_8", "fetch", batch=4, q="whole", kv_max=16384, spread=0.3, page=64),
        # a step of a busy server with a 4-bit cache: many requests of very different lengths, one slot of the batch idle
        _case("step_ragged_4", "attend", bits=4, batch=32, kv_max=16384, spread=0.95, idle=True),
        # four requests of 128K tokens in an 8-bit cache, 64 query heads on 8 kv-heads
        _case("step_128k_8", "attend", hq=64, batch=4, kv_max=131071, page=64),
        # a chunk of two long prompts over an 8-bit cache
        _case("chunk_16k_8", "attend", batch=2, q="all", q_max=2048, kv_max=16384, page=64),
        # the smallest call: one token of a small model that looks at its last 128 rows and four first ones
        _case("window_step_small", "attend", bits=16, dtype="fp16", hq=8, hkv=2, d=64, kv_max=2049, window=128, sink=4),
        # a step of long requests of a model whose layers look 4096 rows back
        _case("window_step_32k", "attend", bits=16, batch=16, kv_max=32768, spread=0.4, window=4096, sink=4),
        # chunks of two long prompts under a window, odd lengths; capped scores
        _case("window_chunk", "attend", bits=16, batch=2, q="ragged", q_max=2049, kv_max=16001, spread=0.2, window=1024, sink=4, cap=50.0),
        # one request's 25 drafted tokens
        _case("tree_small", "attend", bits=16, q="all", q_max=25, kv_max=2100, tree=True),
        # trees of up to 64 drafted tokens of eight requests over an 8-bit cache
        _case("tree_batch_8", "attend", batch=8, q="ragged", q_max=64, kv_max=8192, spread=0.5, tree=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "fetch", "attend", "attend", "attend", "attend"])
    hkv, g = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 3, 4, 8])
    while hkv * g > 64:
        g = rng.choice([1, 2, 3, 4])
    d = rng.choice([64, 128])
    kw = dict(dtype=rng.choice(["bf16", "fp16"]), hkv=hkv, hq=hkv * g, d=d, page=rng.choice([16, 16, 32, 64, 128]),
              batch=_log(rng, 1, 32), spread=rng.choice([0.0, 0.3, 0.6, 0.95]), lens=rng.randrange(1 << 30))
    if kind == "store":
        q = rng.choice(["one", "ragged", "mixed", "all"])
        q_max = 1 if q == "one" else _log(rng, 2, min(4096, 8192 * 48 // ((hkv * g + 2 * hkv) * kw["batch"])))
        return _case(None, kind, bits=rng.choice([8, 4]), q=q, q_max=q_max, kv_max=q_max + _log(rng, 1, 8192), axes=rng.choice([1, 2, 3]),
                     rot=rng.choice([d, d, d // 2]), adjacent=rng.random() < 0.3, **kw)
    if kind == "fetch":
        return _case(None, kind, bits=rng.choice([8, 4]), q="whole", kv_max=_log(rng, 1, min(32768, 4 * 16384 * 8 * 128 // (hkv * d * kw["batch"]))), **kw)
    rows = 4 * 131072 * 8 * 128 // (hkv * d)                # of all sequences: what the largest listed cache holds
    look = rng.choice(["all", "window", "window", "tree", "tree"])
    kw["bits"] = rng.choice([8, 4]) if look == "all" else rng.choice([16, 8, 4])
    if look == "tree":
        q, q_max = rng.choice(["all", "ragged", "ragged", "mixed"]), _log(rng, 2, 200)
    else:
        q = rng.choice(["one", "one", "mixed", "ragged", "all"])
        q_max = 1
    if q == "one":
        kv_max = _log(rng, 16, min(131072, max(17, rows // (2 * kw["batch"]))))
    else:
        pairs = 2 * 2048 * 16384 * 32 // (2 * hkv * g * kw["batch"])     # half the largest listed case's scores
        if look != "tree":
            q_max = _log(rng, 2, min(2048, max(3, pairs // 64)))
        kv_max = q_max + _log(rng, 1, max(2, min(16384, pairs // q_max)))
    if look != "all" and (look == "window" or rng.random() < 0.3):
        kw.update(window=_log(rng, 1, 8192), sink=rng.choice([0, 1, 4, 64]))
    return _case(None, kind, q=q, q_max=q_max, kv_max=kv_max, tree=look == "tree", cap=rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]),
                 idle=kw["batch"] > 2 and rng.random() < 0.3, **kw)


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
        elif c["q"] == "whole":
            n = max(1, int(c["kv_max"] * f))
        else:
            n = max(1, int(c["q_max"] * (1.0 if b == 0 else 1.0 - 0.8 * r.random())))
        if c["idle"] and b == c["batch"] - 1:
            n, t = 0, 0
        else:
            t = n if c["q"] == "whole" else max(n, int(c["kv_max"] * f))
        q.append(n)
        kv.append(t)
    return q, kv


def _drafts(c, seed):
    """Every sequence's drafted tokens: the set of tokens (as a number's bits) that each sees, a few branches at each."""
    r = random.Random(seed * 31 + 5)
    trees = []
    for n in _lengths(c)[0]:
        seen = []
        for i in range(n):
            up = r.randrange(max(0, i - 6), i) if i else -1
            seen.append((seen[up] if up >= 0 else 0) | 1 << i)
        trees.append(seen)
    return trees


# ---- packed rows, plain -----------------------------------------------------------------------

def _power(e, like):
    """2^e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64).to(like.dtype)


def _exponent(y, bias):
    return torch.where(y == 0, 1 - bias, torch.frexp(y).exponent - 1).clamp(min=1 - bias)


def _split(x, bits):
    """Codes' values and blocks' scale bytes of rows [..., d], in x's precision (plain: 64 bits next to the codes' borders)."""
    bias, frac, top = FORMS[bits]
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(blocks.abs().amax(-1))                                          # m in [1/2, 1)
    first = torch.tensor(top, dtype=x.dtype, device=x.device).frexp()
    s = (e - first.exponent + (m > first.mantissa).int()).clamp(min=-126)
    s = torch.where(m == 0, torch.full_like(s, -126), s)
    y = blocks * _power(-s[..., None], blocks)
    step = _exponent(y, bias) - frac
    y = (y * _power(-step, y)).round() * _power(step, y)
    return y.reshape(x.shape), (s + 127).to(torch.uint8)


def _codes(y, bits):
    """Bytes [..., d * bits / 8] of codes' values."""
    bias, frac, _ = FORMS[bits]
    e = _exponent(y, bias)
    whole = (y.abs() * _power(frac - e, y)).int() + (e + bias - 1) * (1 << frac)        # the implicit bit counts the exponent up
    code = whole + (torch.signbit(y).int() << bits - 1)
    if bits == 4:
        code = code[..., 0::2] + code[..., 1::2] * 16
    return code.to(torch.uint8)


def _values(bits, device):
    bias, frac, _ = FORMS[bits]
    c = torch.arange(1 << bits, device=device)
    e, m = (c >> frac) & (1 << bits - 1 - frac) - 1, (c & (1 << frac) - 1).float()
    y = torch.where(e > 0, m + (1 << frac), 2 * m) * _power(e - bias - frac, m)
    return torch.where(c >> bits - 1 > 0, -y, y)


def _unpack(codes, scale, bits):
    """Rows [..., d] of packed ones, in 32 bits."""
    if bits == 8:
        y = codes.view(torch.float8_e4m3fn).float()
    else:
        y = _values(4, codes.device)[torch.stack([codes & 15, codes >> 4], -1).int()].reshape(*codes.shape[:-1], -1)
    return (y.reshape(*scale.shape, 32) * (scale.int() << 23).view(torch.float32)[..., None]).reshape(y.shape)


# ---- what a program has in hand ------------------------------------------------------------------

def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 29)
    dt = DTYPES[c["dtype"]]
    B, hq, hkv, d, ps, bits = c["batch"], c["hq"], c["hkv"], c["d"], c["page"], c["bits"]
    q_len, kv_len = _lengths(c)
    need = [-(-t // ps) for t in kv_len]
    n_pages = sum(need) + 3
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
    first = table[:, 0][table[:, 0] >= 0].long()
    for name in ("k", "v"):
        x = normal(n_pages, hkv, ps, d)
        if name == "k":
            x *= lift
            x[first, :, :4] *= 2.0
        if bits == 16:
            s[name] = x.to(dt)
        else:
            y, s[name + "_scale"] = _split(x.to(dt).float(), bits)
            s[name] = _codes(y, bits)
    s["pos"] = torch.full((n_pages, hkv, ps), -1, dtype=torch.int32, device=dev)
    fused = normal(n, hq + 2 * hkv, d)                                                 # a fused projection's output
    if c["kind"] == "attend":
        # heads differ in how sharply they look
        fused[:, :hq] *= torch.where(torch.rand(hq, generator=g, device=dev) < 0.5, 0.6, 1.8)[None, :, None]
    fused = fused.to(dt)
    s["q"], s["new_k"], s["new_v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    if c["kind"] == "attend":
        s["scale"] = 1.0 / math.sqrt(d)
        s["out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
        s["lse"] = torch.empty((n, hq), dtype=torch.float32, device=dev)
        if c["tree"]:
            words = -(-s["max_q"] // 64)
            bits_of = [[x >> 64 * w & (1 << 64) - 1 for w in range(words)] for seen in _drafts(c, int(seed)) for x in seen]
            s["tree"] = torch.tensor([[w - (1 << 64) if w >> 63 else w for w in x] for x in bits_of], dtype=torch.int64, device=dev)
    if c["kind"] != "attend":
        s["k_read"], s["v_read"] = torch.empty((n, hkv, d), dtype=dt, device=dev), torch.empty((n, hkv, d), dtype=dt, device=dev)
    if c["kind"] == "store":
        s["q_out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
        shift = [int(x) for x in torch.randint(0, 30000, (B,), generator=g, device=dev)]
        base = torch.cat([torch.arange(t - a, t, device=dev, dtype=torch.int32) + z for a, t, z in zip(q_len, kv_len, shift)])
        grid = [base, base % 27, base // 27 % 31]                                      # time, height, width
        s["positions"] = torch.stack(grid[:c["axes"]]).contiguous()
        half = c["rot"] // 2
        s["freq"] = 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        s["axis"] = [0] * half if c["axes"] == 1 else [min(c["axes"] - 1, i * c["axes"] // half) for i in range(half)]
        s["axis_dev"] = torch.tensor(s["axis"], device=dev)
    if own:
        from paper_2603_08727_amd import paged as P
        s["batch"] = P.arkv_page_batch(s["cu_q"], s["kv_len"], s["table"], n, s["max_q"], s["max_kv"])
        if bits == 16:
            s["pages"] = P.arkv_pages(s["k"], s["v"], s["pos"])
            s["workspace"] = P.arkv_paged_workspace(s["pages"], s["batch"], hq)
        else:
            s["pages"] = P.arkv_packed_pages(s["k"], s["v"], s["k_scale"], s["v_scale"], s["pos"], dt)
            s["workspace"] = P.arkv_packed_workspace(s["pages"], s["batch"], hq)
        s["sight"] = P.arkv_sight(c["window"], c["sink"], s.get("tree")) if c["window"] or c["tree"] else None
        if c["kind"] == "store":
            s["rotary"] = P.arkv_rotary(s["freq"], s["axis"], c["axes"], adjacent=c["adjacent"])
    return s


# ---- plain forms ------------------------------------------------------------------------------

def _tokens(s):
    """Sequence of every new token, and its index among that sequence's new ones."""
    t = torch.arange(s["n"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu_q"][1:].contiguous(), t, right=True)
    return b, t - s["cu_q"][b]


def _places(s):
    """Page and offset of every new token's row."""
    ps = s["case"]["page"]
    b, i = _tokens(s)
    slot = s["kv_len"][b] - (s["cu_q"][b + 1] - s["cu_q"][b]) + i
    return s["table"][b, (slot // ps).long()].long(), (slot % ps).long()


def _fetch(s):
    page, off = _places(s)
    bits, dt = s["case"]["bits"], s["k_read"].dtype
    return {x: _unpack(s[x][page, :, off], s[x + "_scale"][page, :, off], bits).to(dt) for x in ("k", "v")}


def _store(s):
    c = s["case"]
    half = c["rot"] // 2
    angle = s["positions"][s["axis_dev"]].double() * s["freq"][:, None]                # [half][n]
    cos, sin = angle.cos().t()[:, None], angle.sin().t()[:, None]

    def turned(x):
        y, cs, sn = x.clone(), cos.to(x.dtype), sin.to(x.dtype)
        if c["adjacent"]:
            a, e = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cs - e * sn, e * cs + a * sn
        else:
            a, e = x[..., :half], x[..., half:2 * half]
            y[..., :half], y[..., half:2 * half] = a * cs - e * sn, e * cs + a * sn
        return y

    page, off = _places(s)
    for name, x in (("k", turned(s["new_k"].double())), ("v", s["new_v"].double())):   # (64 bits: turned keys next to a border of codes)
        y, scale = _split(x, c["bits"])
        s[name][page, :, off] = _codes(y, c["bits"])
        s[name + "_scale"][page, :, off] = scale
    s["pos"][page, :, off] = s["positions"][0][:, None].expand(-1, c["hkv"])
    return {"q": turned(s["q"].float()).to(s["q_out"].dtype), **_fetch(s), "pos": s["pos"]}


def _dense(s, name):
    """[B][kv-head][slot][channel] of a pool, in 32 bits."""
    c = s["case"]
    page = s["table"].clamp(min=0).long()
    x = s[name][page].float() if c["bits"] == 16 else _unpack(s[name][page], s[name + "_scale"][page], c["bits"])
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, c["d"])[:, :, :s["max_kv"]]


def _seen(s):
    """[B][new token][slot]"""
    c = s["case"]
    q_len = s["cu_q"][1:] - s["cu_q"][:-1]
    i, j = torch.arange(s["max_q"], device="cuda"), torch.arange(s["max_kv"], device="cuda")
    ctx = (s["kv_len"] - q_len)[:, None]
    place = ctx + i
    if c["tree"]:
        t = (s["cu_q"][:-1, None] + i).clamp(max=s["n"] - 1)
        drawn = s["tree"][t]                                                           # [B][new][word]
        above = (drawn[..., i // 64] >> (i % 64) & 1).bool() & (i < q_len[:, None])[:, None]
        place = ctx + (above.sum(-1) - 1).clamp(min=0)
    old = j <= place[..., None] if not c["tree"] else (j < ctx)[:, None]
    if c["window"]:
        old = old & ((j > place[..., None] - c["window"]) | (j < c["sink"]))
    if c["tree"]:
        new = j - ctx                                                                  # [B][slot]
        hit = above.gather(2, new.clamp(0, s["max_q"] - 1)[:, None].expand(-1, s["max_q"], -1))
        old = old | hit & ((new >= 0) & (new < q_len[:, None]))[:, None]
    return old & (j < s["kv_len"][:, None])[:, None]


def _attend(s):
    c = s["case"]
    B, hq, hkv, d, mq, mk = c["batch"], c["hq"], c["hkv"], c["d"], s["max_q"], s["max_kv"]
    i = torch.arange(mq, device="cuda")
    tok = (s["cu_q"][:-1, None] + i).clamp(max=s["n"] - 1)
    q = s["q"][tok].float().permute(0, 2, 1, 3).reshape(B, hkv, hq // hkv * mq, d)
    x = torch.matmul(q, _dense(s, "k").transpose(2, 3).contiguous()).mul_(s["scale"])
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    x.reshape(B, hkv, hq // hkv, mq, mk).masked_fill_(~_seen(s)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, _dense(s, "v").contiguous()) / total
    lse = top + total.log()
    b, i = _tokens(s)
    out = out.reshape(B, hq, mq, d)[b, :, i.long()]
    return {"out": out.to(s["out"].dtype), "lse": lse.reshape(B, hq, mq)[b, :, i.long()]}


def run(s):
    c = s["case"]
    if not own:
        return {"store": _store, "fetch": _fetch, "attend": _attend}[c["kind"]](s)
    from paper_2603_08727_amd import paged as P
    if c["kind"] == "attend":
        if c["bits"] == 16:
            P.arkv_paged_attention_sight(s["pages"], s["batch"], s["sight"], s["q"], s["scale"], s["out"], lse=s["lse"], cap=c["cap"],
                                         workspace=s["workspace"])
        else:
            P.arkv_packed_attention(s["pages"], s["batch"], s["q"], s["scale"], s["out"], lse=s["lse"], cap=c["cap"], sight=s["sight"],
                                    workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "store":
        P.arkv_packed_append(s["pages"], s["batch"], s["rotary"], s["q"], s["new_k"], s["new_v"], s["positions"], s["q_out"])
    P.arkv_packed_read(s["pages"], s["batch"], s["k_read"], s["v_read"])
    out = {"k": s["k_read"], "v": s["v_read"]}
    return out if c["kind"] == "fetch" else {"q": s["q_out"], "pos": s["pos"], **out}


# ---- what a pass cannot do without ------------------------------------------------------------

def _pairs(c):
    """Of every sequence: (new token, slot) pairs that are seen, and rows that some token sees."""
    got = []
    trees = _drafts(c, 0) if c["tree"] else None
    for b, (a, t) in enumerate(zip(*_lengths(c))):
        ctx, w = t - a, c["window"] or t
        pairs, least = 0, t
        for i in range(a):
            p = ctx + (bin(trees[b][i]).count("1") - 1 if c["tree"] else i)
            lo = max(0, p - w + 1)
            end = ctx if c["tree"] else p + 1
            pairs += max(0, end - lo) + min(c["sink"], lo, end) + (bin(trees[b][i]).count("1") if c["tree"] else 0)
            least = min(least, lo)
        got.append((pairs, t - least + min(c["sink"], least) if a else 0))
    return got


def work(case):
    c = case
    q_len, kv_len = _lengths(c)
    n, d, hq, hkv = sum(q_len), c["d"], c["hq"], c["hkv"]
    row = 2 * d if c["bits"] == 16 else d * c["bits"] // 8 + d // 32                   # of a key or a value
    pages = sum(-(-t // c["page"]) for t in kv_len)
    meta = 4 * (2 * c["batch"] + 1)
    if c["kind"] == "store":
        # written once, and what was written read once
        return {"bytes": n * (2 * (2 * hq + 2 * hkv) * d + 2 * hkv * (2 * row + 2 * d) + 4 * hkv + 4 * c["axes"]) + meta, "flops": 3.0 * n * (hq + hkv) * c["rot"]}
    if c["kind"] == "fetch":
        return {"bytes": n * 2 * hkv * (row + 2 * d) + meta + 4 * pages, "flops": float(n * 2 * hkv * d)}
    pairs = _pairs(c)
    rows = sum(r for _, r in pairs)
    drawn = 8 * n * -(-max(q_len) // 64) if c["tree"] else 0
    return {"bytes": rows * hkv * 2 * row + n * hq * (4 * d + 4) + meta + 4 * -(-rows // c["page"]) + drawn,
            "flops": 4.0 * d * sum(p for p, _ in pairs) * hq}


# ---- the same in 64 bits ------------------------------------------------------------------------

def _table(bits):
    """Every code's value, by the format's definition."""
    bias, frac, _ = FORMS[bits]
    got = []
    for code in range(1 << bits):
        e, m = code >> frac & (1 << bits - 1 - frac) - 1, code & (1 << frac) - 1
        x = math.ldexp(m, 1 - bias - frac) if e == 0 else math.ldexp((1 << frac) + m, e - bias - frac)
        got.append(-x if code >> bits - 1 else x)
    return got


def _exact_unpack(codes, scale, bits):
    t = torch.tensor(_table(bits), dtype=torch.float64, device=codes.device)
    if bits == 8:
        t[[0x7F, 0xFF]] = math.nan
        y = t[codes.int()]
    else:
        y = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
        y[..., 0::2], y[..., 1::2] = t[(codes % 16).int()], t[(codes // 16).int()]
    return y * _power(scale.long() - 127, y).repeat_interleave(32, -1)


def _exact_packed(x, bits):
    """The values that packed rows of x stand for: in every block the scale by trial, the code by the borders between codes."""
    up = [v for v in _table(bits)[:1 << bits - 1] if v <= FORMS[bits][2]]
    border = torch.tensor([(a + b) / 2 for a, b in zip(up, up[1:])], dtype=torch.float64, device=x.device)
    value = torch.tensor(up, dtype=torch.float64, device=x.device)
    y = x.reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    s = torch.ceil(torch.log2(top / up[-1])).clamp(min=-126.0).nan_to_num(neginf=-126.0)
    s = torch.where(top > up[-1] * _power(s, y), s + 1, s)
    s = torch.where((top <= up[-1] * _power(s - 1, y)) & (s > -126), s - 1, s)
    z = y.abs() / _power(s, y)
    i = torch.bucketize(z, border)                                                     # a border counts to the code below
    i = i + ((i < len(up) - 1) & (i % 2 == 1) & (z == border[i.clamp(max=len(up) - 2)])).long()
    return (torch.sign(y) * value[i] * _power(s, y)).reshape(x.shape)


def _rows_of(s, name, b, t):
    """[kv-head][t][...] of a sequence's slots, in slot order."""
    pages = [int(x) for x in s["table"][b, :-(-t // s["case"]["page"])].tolist()]
    return torch.cat([s[name][p] for p in pages], dim=1)[:, :t]


def _exact_rows(s, name, b, t):
    x = _rows_of(s, name, b, t)
    return x if s["case"]["bits"] == 16 else _exact_unpack(x, _rows_of(s, name + "_scale", b, t), s["case"]["bits"]).float()   # (codes' values fit 32 bits)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    q_len, kv_len = _lengths(c)
    n, hq, hkv, d, ps = s["n"], c["hq"], c["hkv"], c["d"], c["page"]
    if c["kind"] == "fetch":
        return {x: torch.cat([_exact_rows(s, x, b, t).transpose(0, 1).double() for b, t in enumerate(kv_len) if t]) for x in ("k", "v")}
    if c["kind"] == "store":
        half = c["rot"] // 2
        first = [2 * i if c["adjacent"] else i for i in range(half)]
        second = [2 * i + 1 if c["adjacent"] else i + half for i in range(half)]
        pos = s["positions"].double()
        turn = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"),
                           torch.stack([pos[ax] * s["freq"][i] for i, ax in enumerate(s["axis"])], dim=1))
        q, k = s["q"].double().clone(), s["new_k"].double().clone()
        for x in (q, k):
            z = torch.complex(x[..., first], x[..., second]) * turn[:, None, :]
            x[..., first], x[..., second] = z.real, z.imag
        held = s["pos"].clone()
        at = 0
        for b, (a, t) in enumerate(zip(q_len, kv_len)):
            slot = torch.arange(t - a, t, device="cuda")
            held[s["table"][b][slot // ps].long(), :, slot % ps] = s["positions"][0, at:at + a, None].expand(-1, hkv)
            at += a
        return {"q": q, "k": _exact_packed(k, c["bits"]), "v": _exact_packed(s["new_v"].double(), c["bits"]), "pos": held}
    out = torch.zeros((n, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((n, hq), dtype=torch.float64, device="cuda")
    trees = _drafts(c, int(seed)) if c["tree"] else None
    at = 0
    for b, (a, t) in enumerate(zip(q_len, kv_len)):
        if not t:
            continue
        ctx = t - a
        see = torch.zeros(a, t, dtype=torch.bool)
        for i in range(a):
            p = ctx + (bin(trees[b][i]).count("1") - 1 if c["tree"] else i)
            see[i, :ctx if c["tree"] else p + 1] = True
            if c["window"]:
                see[i, min(t, c["sink"]):max(c["sink"], p - c["window"] + 1)] = False
            if c["tree"]:
                see[i, ctx:] = torch.tensor([bool(trees[b][i] >> e & 1) for e in range(a)])
        see = see.cuda()
        k, v = _exact_rows(s, "k", b, t), _exact_rows(s, "v", b, t)
        for h in range(hq):
            x = (s["q"][at:at + a, h].double() @ k[h * hkv // hq].double().t()) * s["scale"]
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            x = torch.where(see, x, torch.full_like(x, -math.inf))
            z = torch.logsumexp(x, dim=1)
            out[at:at + a, h] = torch.exp(x - z[:, None]) @ v[h * hkv // hq].double()
            lse[at:at + a, h] = z
        at += a
    return {"out": out, "lse": lse}
