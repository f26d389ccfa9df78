"""Plain 64-bit forms of the operators around a paged cache, one sequence and head at a time, and the error bounds that the
tests allow.  Every bound is derived from the arithmetic: u = half a step of the stored type (bf16 2^-8, fp16 2^-11), fp32
roundings 2^-24 each.
"""
import math
from types import SimpleNamespace

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F32 = 2.0 ** -24


def problem(dev, dtype=torch.bfloat16, hq=8, hkv=2, d=64, page=16, q_len=(1,), kv_len=(40,), seed=0, spare_pages=2, extra_tokens=0,
            hot=2.0, fused=False, width=None, shared=None):
    """Pages, table and new tokens of random sequences; unused slots and pages hold NaN."""
    g = torch.Generator().manual_seed(seed)
    B = len(q_len)
    need = [-(-t // page) for t in kv_len]
    n_pages = sum(need) + spare_pages
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    width = width or max(max(need), 1)
    table = torch.full((B, width), -7, dtype=torch.int32)
    k = torch.full((n_pages, hkv, page, d), math.nan)
    v = torch.full((n_pages, hkv, page, d), math.nan)
    pos = torch.full((n_pages, hkv, page), -1, dtype=torch.int32)
    weight = torch.full((n_pages, hkv, page), math.nan)
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for i in range(need[b]):
            m = min(page, kv_len[b] - i * page)
            p = int(table[b, i])
            k[p, :, :m] = torch.randn(hkv, m, d, generator=g)
            v[p, :, :m] = torch.randn(hkv, m, d, generator=g)
            pos[p, :, :m] = torch.arange(i * page, i * page + m, dtype=torch.int32) * 2
            weight[p, :, :m] = torch.rand(hkv, m, generator=g)
    n = sum(q_len) + extra_tokens
    cu = torch.tensor([sum(q_len[:b]) for b in range(B + 1)], dtype=torch.int32)
    if fused:
        q = torch.randn(n, hq + 2 * hkv, d, generator=g)[:, :hq]
    else:
        q = torch.randn(n, hq, d, generator=g)
    q = (q * hot)
    s = SimpleNamespace(dtype=dtype, hq=hq, hkv=hkv, d=d, page=page, q_len=list(q_len), kv_len_list=list(kv_len), n=n, B=B, n_pages=n_pages)
    full = torch.empty((n, hq + 2 * hkv, d) if fused else (n, hq, d), dtype=dtype)
    full[:, :hq] = q.to(dtype)
    s.q = full.to(dev)[:, :hq]
    s.k, s.v, s.pos, s.weight = k.to(dtype).to(dev), v.to(dtype).to(dev), pos.to(dev), weight.to(dev)
    s.cu_q, s.kv_len, s.table = cu.to(dev), torch.tensor(list(kv_len), dtype=torch.int32).to(dev), table.to(dev)
    s.max_q, s.max_kv = max(max(q_len), 0), max(kv_len)
    s.scale = 1.0 / math.sqrt(d)
    s.spare = order[at:].tolist()
    return s


def rows(s, x, b, h):
    """A pool's rows of sequence b, head h in slot order, and which of them exist."""
    t = min(s.kv_len_list[b], s.table.shape[1] * s.page)
    slot = torch.arange(t, device=s.table.device)
    page = s.table[b].long()[slot // s.page]
    real = (page >= 0) & (page < s.n_pages)
    return x[page.clamp(0, s.n_pages - 1), h, slot % s.page], real


def visible(s, b, prefix=None):
    t, a = s.kv_len_list[b], s.q_len[b]
    slot, i = torch.arange(t, device=s.table.device), torch.arange(a, device=s.table.device)
    see = slot[None] <= (t - a + i)[:, None]
    if prefix is not None:
        see = see | (slot[None] < int(prefix[b]))
    return see & rows(s, s.pos, b, 0)[1][None]


def logits(s, b, hq, cap=0.0, slopes=None, q_pos=None, prefix=None):
    """(x [q][t] with -inf where unseen, largest error an fp32 logit may have)."""
    h = hq // (s.hq // s.hkv)
    at, a = sum(s.q_len[:b]), s.q_len[b]
    see = visible(s, b, prefix)
    k = rows(s, s.k, b, h)[0].double()
    k = torch.where(see.any(0)[:, None], k, torch.zeros_like(k))
    q = s.q[at:at + a, hq].double()
    x = q @ k.t() * s.scale
    size = (q.abs() @ k.abs().t()) * abs(s.scale)
    size = torch.where(see, size, torch.zeros_like(size))
    err = (s.d + 8) * F32 * float(size.max()) if size.numel() else 0.0
    if cap:
        x = cap * torch.tanh(x / cap)
        err += cap * 8 * F32
    if slopes is not None:
        far = (q_pos[at:at + a].double()[:, None] - rows(s, s.pos, b, h)[0].double()[None]).abs()
        x = x - slopes[hq].double() * far
        far = torch.where(see, far, torch.zeros_like(far))
        err += 3 * F32 * float((slopes[hq].double() * far).abs().max()) if far.numel() else 0.0
    return torch.where(see, x, torch.full_like(x, -math.inf)), err


def attention(s, **kw):
    """out, lse and how far each may be off."""
    dev = s.table.device
    out = torch.zeros(s.n, s.hq, s.d, dtype=torch.float64, device=dev)
    lse = torch.full((s.n, s.hq), -math.inf, dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u = U[s.dtype]
    for b in range(s.B):
        at, a = sum(s.q_len[:b]), s.q_len[b]
        if not a or not s.kv_len_list[b]:
            continue
        see = visible(s, b, kw.get("prefix"))
        for hq in range(s.hq):
            x, err = logits(s, b, hq, **kw)
            v = rows(s, s.v, b, hq // (s.hq // s.hkv))[0].double()
            v = torch.where(see.any(0)[:, None], v, torch.zeros_like(v))
            z = torch.logsumexp(x, 1)
            p = torch.where(see, torch.exp(x - z[:, None]), torch.zeros_like(x))
            bad = ~torch.isfinite(v)                   # values that are not finite count for those who see them only
            o = p @ torch.where(bad, torch.zeros_like(v), v)
            if bad.any():
                for j in bad.any(1).nonzero()[:, 0].tolist():
                    seen_by = see[:, j]
                    o[seen_by] += p[seen_by, j, None] * torch.where(bad[j], v[j], torch.zeros_like(v[j]))[None]
            out[at:at + a, hq], lse[at:at + a, hq] = o, z
            va = torch.where(bad, torch.zeros_like(v), v).abs()
            # probabilities: rounded once (u), logit error in numerator and denominator, sums of t terms in fp32
            t = p @ va
            tol[at:at + a, hq] = u * o.abs() + (u + 2 * err + 64 * F32 + 2 * math.sqrt(x.shape[1]) * F32) * t + 1e-30
            if s.dtype == torch.float16:
                # below 2^-14 of the softmax reference fp16 probabilities are off by up to 2^-25 each; outputs by 2^-25
                tol[at:at + a, hq] += 2.0 ** -25 * (see.double() @ va) * torch.exp(x.amax(1) - z)[:, None].nan_to_num(0.0) + 2.0 ** -25
            ltol[at:at + a, hq] = err + 16 * F32 * (1 + z.abs().nan_to_num(0.0, posinf=0.0, neginf=0.0)) + math.sqrt(x.shape[1]) * F32
    return out, lse, tol, ltol


def close(x, ref, tol, what):
    x = x.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(x), torch.isnan(ref)), f"{what}: NaN in other places"
    inf = ~fine & ~torch.isnan(ref)
    assert torch.equal(x[inf], ref[inf]), f"{what}: infinities differ"
    over = ((x - ref).abs() / tol.clamp(min=1e-300))[fine]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times the allowed error"
    return worst


def weights(s, lse, decay, carried, **kw):
    """weight of every slot in use, and the allowed error; others as they are."""
    out = s.weight.double().clone()
    tol = torch.zeros_like(out)
    G = s.hq // s.hkv
    for b in range(s.B):
        at, a, t = sum(s.q_len[:b]), s.q_len[b], s.kv_len_list[b]
        if not t:
            continue
        see = visible(s, b, kw.get("prefix"))
        slot = torch.arange(t, device=s.table.device)
        for h in range(s.hkv):
            total, rel = torch.zeros(t, dtype=torch.float64, device=s.table.device), 0.0
            for hq in range(h * G, (h + 1) * G):
                x, err = logits(s, b, hq, **kw)
                p = torch.where(see, torch.exp(x - lse[at:at + a, hq].double()[:, None]), torch.zeros_like(x))
                total += p.sum(0)
                rel = max(rel, err + F32 * 8 * (1 + float(x[see].abs().max()) if see.any() else 1.0))
            page = s.table[b].long()[slot // s.page]
            real = (page >= 0) & (page < s.n_pages)
            page, off = page[real], (slot % s.page)[real]
            old = carried[page, h, off].double() * decay if decay else torch.zeros_like(total[real])
            out[page, h, off] = old + total[real]
            tol[page, h, off] = (2 * rel + (32 + math.sqrt(a * G)) * F32) * total[real] + 2 * F32 * (old.abs() + total[real]) + 1e-37
    return out, tol


def evict(s, keep, sink, recent, max_keep):
    """kept [B][H][max_keep] and new lengths."""
    kept = torch.full((s.B, s.hkv, max_keep), -1, dtype=torch.int32)
    lens = []
    for b in range(s.B):
        t = s.kv_len_list[b]
        m = min(t, max(0, min(int(keep[b]), max_keep)))
        f = min(sink, m)
        r = min(recent, m - f)
        lens.append(m)
        for h in range(s.hkv):
            w, real = rows(s, s.weight, b, h)
            w = [float(x) if ok and x == x else None for x, ok in zip(w.cpu().tolist(), real.cpu().tolist())]
            ranked = sorted(range(f, t - r), key=lambda j: (w[j] is None, -(w[j] if w[j] is not None else 0.0), j))
            stay = sorted(list(range(f)) + ranked[:m - f - r] + list(range(t - r, t)))
            kept[b, h, :m] = torch.tensor(stay, dtype=torch.int32)
    return kept, lens


def rotate(x, positions, freq, axis, adjacent):
    """[n][heads][d] in 64 bits, and the allowed error of an fp32 rotation stored with one rounding."""
    half = freq.numel()
    y = x.double().clone()
    tol = torch.zeros_like(y)
    u = U[x.dtype]
    for i in range(half):
        a, e = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        t = positions[axis[i]].double() * freq[i].double()
        c, sn = torch.cos(t)[:, None], torch.sin(t)[:, None]
        xa, xe = x[..., a].double(), x[..., e].double()
        y[..., a], y[..., e] = xa * c - xe * sn, xe * c + xa * sn
        # sine and cosine to 4 fp32 steps of 1, two products, one sum
        slack = 8 * F32 * 2 * (xa.abs() + xe.abs())
        tol[..., a] = slack + u * (y[..., a].abs() + slack)
        tol[..., e] = slack + u * (y[..., e].abs() + slack)
    if x.dtype == torch.float16:
        tol[..., :2 * half] += 2.0 ** -25
    return y, tol
