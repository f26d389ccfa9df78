"""Plain 64-bit forms of packed rows and of limited sight, and problems with packed pages.  Attention over them is
paged_ref.attention's: what packed rows stand for is exact in the rows' type, so its bounds hold as they are."""
import math
from types import SimpleNamespace
from unittest import mock

import torch

import paged_ref as R

FORMS = {8: (4, 3, 448.0), 4: (2, 1, 6.0)}             # bits: of exponent, of mantissa, largest value
LIMIT = {torch.bfloat16: float(torch.finfo(torch.bfloat16).max), torch.float16: 65504.0}


def table(bits):
    """What every code stands for."""
    ex, frac, _ = FORMS[bits]
    bias, got = (1 << ex - 1) - 1, []
    for code in range(1 << bits):
        e, m = (code >> frac) % (1 << ex), code % (1 << frac)
        x = m * 2.0 ** (1 - bias - frac) if e == 0 else ((1 << frac) + m) * 2.0 ** (e - bias - frac)
        if bits == 8 and code % 128 == 127:
            x = math.nan
        got.append(-x if code >> bits - 1 else x)
    return torch.tensor(got, dtype=torch.float64)


def values(codes, scale, bits):
    """[..., d] in 64 bits (CPU tensors)."""
    t = table(bits)
    if bits == 8:
        y = t[codes.long()]
    else:
        y = torch.stack([t[(codes & 15).long()], t[(codes >> 4).long()]], -1).reshape(*codes.shape[:-1], -1)
    s = torch.where(scale == 255, torch.full(scale.shape, math.nan, dtype=torch.float64), torch.ldexp(torch.ones(scale.shape, dtype=torch.float64), scale.int() - 127))
    return y * s.repeat_interleave(32, -1)


def pack(x, bits, dtype):
    """Codes and scale bytes of rows x [..., d] (64 bits, CPU) as the header defines them, one block at a time."""
    ex, frac, top = FORMS[bits]
    up = table(bits)[:1 << bits - 1]
    up = up[up <= top]
    border = (up[1:] + up[:-1]) / 2
    rows = x.reshape(-1, 32)
    codes, scales = torch.zeros(rows.shape, dtype=torch.int64), torch.zeros(len(rows), dtype=torch.int64)
    for r, row in enumerate(rows):
        fine = row.abs() <= LIMIT[dtype]
        most = float(row[fine].abs().max()) if fine.any() else 0.0
        s = 1
        if most > 0:
            s = max(1, math.frexp(most)[1] + 127 - math.frexp(top)[1] - 1)
            while most > math.ldexp(top, s - 127):
                s += 1
        y = row.abs() * math.ldexp(1.0, 127 - s)
        i = torch.bucketize(y, border)                 # nearest; a border counts to the code below
        tie = (i < len(border)) & (y == border[i.clamp(max=len(border) - 1)])
        i = torch.where(tie & (i % 2 == 1), i + 1, i)
        last = max(c for c in range(len(up)) if math.ldexp(float(up[c]), s - 127) <= LIMIT[dtype])
        i = i.clamp(max=last)
        i = torch.where(torch.signbit(row), i + (1 << bits - 1), i)
        if bits == 8:
            i = torch.where(fine, i, torch.full_like(i, 127))
        elif not fine.all():
            s = 255
        codes[r], scales[r] = i, s
    codes = codes.reshape(x.shape)
    if bits == 4:
        codes = codes[..., 0::2] + 16 * codes[..., 1::2]
    return codes.to(torch.uint8), scales.reshape(*x.shape[:-1], -1).to(torch.uint8)


def same_values(codes, scale, want_codes, want_scale, bits):
    """Whether rows stand for the same, NaN where NaN."""
    a, b = values(codes.cpu(), scale.cpu(), bits), values(want_codes, want_scale, bits)
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    ok = ~torch.isnan(b)
    assert torch.equal(a[ok], b[ok]), (a[ok] - b[ok]).abs().max()
    assert torch.equal(torch.signbit(a[ok]), torch.signbit(b[ok]))


def quick_pack(x, bits):
    """Some codes and scales near the rows x (fp32): for problems whose rows may be any."""
    ex, frac, top = FORMS[bits]
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    e = torch.frexp(blocks.abs().amax(-1).clamp(min=2.0 ** -100) / top)[1]
    y = blocks / torch.ldexp(torch.ones(e.shape), e)[..., None]
    if bits == 8:
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        codes = ((y[..., None].abs() - table(4)[:8].float()).abs().argmin(-1) + 8 * torch.signbit(y)).to(torch.uint8)
    codes = codes.reshape(x.shape)
    if bits == 4:
        codes = codes[..., 0::2] + 16 * codes[..., 1::2]
    return codes.contiguous(), (e + 127).to(torch.uint8)


def every_pair(bits, d):
    """Rows' bytes [rows][d bits / 8] and scale bytes [rows][d / 32]: every byte of codes in a block of every scale."""
    per = 32 * bits // 8
    codes = torch.arange(256, dtype=torch.int32).reshape(1, -1, per).expand(256, -1, -1)
    scale = torch.arange(256, dtype=torch.int32)[:, None].expand(-1, 256 // per)
    return codes.reshape(-1, d * bits // 8).to(torch.uint8), scale.reshape(-1, d // 32).to(torch.uint8)


def problem(dev, bits, dtype=torch.bfloat16, **kw):
    """paged_ref.problem with packed pages: s.k and s.v are what the codes stand for; unused slots hold NaN."""
    s = R.problem("cpu", dtype, **kw)
    for name in ("k", "v"):
        x = getattr(s, name).float()
        lost = torch.isnan(x)
        codes, scale = quick_pack(torch.where(lost, torch.zeros_like(x), x), bits)
        scale = torch.where(lost.reshape(*scale.shape, 32).any(-1), torch.full_like(scale, 255), scale)
        setattr(s, name, values(codes, scale, bits).to(dtype).to(dev))
        setattr(s, name + "_codes", codes.to(dev))
        setattr(s, name + "_scale", scale.to(dev))
    s.bits = bits
    for name in ("q", "pos", "weight", "cu_q", "kv_len", "table"):
        x = getattr(s, name)
        setattr(s, name, x.to(dev) if name != "q" else strided(x, dev))
    return s


def strided(x, dev):
    """x on dev, with the strides that it has."""
    base = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=dev)
    base.copy_(x)
    return base


def set_value(s, name, page, h, off, ch, nan=True):
    """Makes one channel of a packed row no number (with 4 bits: its block)."""
    if s.bits == 8:
        getattr(s, name + "_codes")[page, h, off, ch] = 127
        getattr(s, name)[page, h, off, ch] = math.nan
    else:
        getattr(s, name + "_scale")[page, h, off, ch // 32] = 255
        getattr(s, name)[page, h, off, ch // 32 * 32:ch // 32 * 32 + 32] = math.nan


def sight(s, b, prefix=None, window=0, sink=0, tree=None):
    """[q][t]: which slots the new tokens of sequence b see.  tree: [n_tokens][max_q] truth values."""
    t, a, at = s.kv_len_list[b], s.q_len[b], sum(s.q_len[:b])
    see = torch.zeros(a, t, dtype=torch.bool)
    for i in range(a):
        p = t - a + i
        if p >= 0:
            if tree is None:
                old = [j for j in range(p + 1)]
            else:
                mine = [bool(x) for x in tree[at + i][:a]]
                old = [j for j in range(max(0, t - a))]
                p = t - a + max(0, sum(mine) - 1)
                for e in range(a):
                    if mine[e] and 0 <= t - a + e:
                        see[i, t - a + e] = True
            if window:
                old = [j for j in old if j > p - window or j < sink]
            see[i, old] = True
        if prefix is not None:
            see[i, :max(0, int(prefix[b]))] = True
    return see.to(s.table.device) & R.rows(s, s.pos, b, 0)[1][None]


def attention(s, window=0, sink=0, tree=None, **kw):
    with mock.patch.object(R, "visible", lambda s, b, prefix=None: sight(s, b, prefix, window, sink, tree)):
        return R.attention(s, **kw)


def words(tree):
    """Truth values [n][m] as int64 words [n][ceil(m / 64)]."""
    n, m = tree.shape
    got = []
    for row in tree.tolist():
        x = sum(1 << e for e, on in enumerate(row) if on)
        got.append([(x >> 64 * w) % (1 << 64) for w in range(max(1, -(-m // 64)))])
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in row] for row in got], dtype=torch.int64)


def drafts(s, seed=0, branch=5):
    """[n][max_q]: every sequence's new tokens as a tree of drafts: ancestors and itself."""
    g = torch.Generator().manual_seed(seed)
    tree = torch.zeros(s.n, max(1, s.max_q), dtype=torch.bool)
    at = 0
    for a in s.q_len:
        for i in range(a):
            if i:
                up = max(0, i - 1 - int(torch.randint(0, branch, (1,), generator=g)))
                tree[at + i] = tree[at + up]
            tree[at + i, i] = True
        at += a
    return tree
