"""The paged cache and the attention over it in 64 bits, from their definitions, on the CPU; bounds that count roundings."""
import math

import torch

# (a module of its own: it shares no code with the package or the measured cases)
TOP = {"e4m3": 448.0, "e2m1": 6.0}
LOWEST = -100


def code_values(fmt):
    """The numbers of the codes without a sign, rising."""
    if fmt == "e2m1":
        return [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    small = [m / 512.0 for m in range(8)]
    return small + [math.ldexp(1.0 + m / 8.0, e - 7) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]


def quantised(x, fmt):
    """(codes as their indexes with the sign's bit on top, exponents) of rows x [..][H]; blocks with a NaN or an infinity: exponent 128, code 0."""
    worth = torch.tensor(code_values(fmt), dtype=torch.float64)
    sign = 128 if fmt == "e4m3" else 8
    H = x.shape[-1]
    codes = torch.zeros(x.shape, dtype=torch.int64)
    exponents = torch.zeros(*x.shape[:-1], -(-H // 32), dtype=torch.int64)
    for n, first in enumerate(range(0, H, 32)):
        y = x[..., first:first + 32].double().cpu()
        fine = torch.isfinite(y).all(-1)
        y = torch.where(fine.unsqueeze(-1), y, torch.zeros_like(y))
        top = y.abs().amax(-1)
        s = torch.full(top.shape, LOWEST, dtype=torch.int64)
        for e in range(LOWEST, 127):                       # the smallest that is enough
            s = torch.where(top > TOP[fmt] * 2.0 ** e, torch.full_like(s, e + 1), s)
        y = y * torch.exp2(-s.double()).unsqueeze(-1)
        a = y.abs()
        code = torch.zeros(a.shape, dtype=torch.int64)
        for i in range(1, len(worth)):
            middle = (worth[i] + worth[i - 1]) / 2
            code = torch.where((a > middle) | ((a == middle) & (i % 2 == 0)), torch.full_like(code, i), code)
        code = code + sign * torch.signbit(y).long()
        codes[..., first:first + 32] = torch.where(fine.unsqueeze(-1), code, torch.zeros_like(code))
        exponents[..., n] = torch.where(fine, s, torch.full_like(s, 128))
    return codes, exponents


def decoded(codes, exponents, fmt):
    worth = torch.tensor(code_values(fmt) + ([math.nan] if fmt == "e4m3" else []), dtype=torch.float64)
    worth = torch.cat([worth, -worth])
    y = worth[codes] * torch.exp2(exponents.double()).repeat_interleave(32, -1)[..., :codes.shape[-1]]
    bad = (exponents == 128).repeat_interleave(32, -1)[..., :codes.shape[-1]]
    y = torch.where(bad, torch.full_like(y, math.nan), y)
    return y.float().double()                             # (2^128 and more: infinite)


def cache_values(cache, i):
    """All of the cache's K (i = 0) or V, [pages][kv_heads][page_rows][H] in 64 bits."""
    x = cache[i].cpu()
    if x.dtype == torch.bfloat16:
        return x.double()
    fmt = "e4m3" if x.dtype == torch.float8_e4m3fn else "e2m1"
    if fmt == "e4m3":
        codes = x.view(torch.uint8).long()
    else:
        codes = torch.stack([x.long() & 15, x.long() >> 4], -1).flatten(-2)
    blocks = -(-codes.shape[-1] // 32)
    return decoded(codes, cache[2 + i].cpu()[..., :blocks].long() - 127, fmt)


def sequence(values, table, b, tokens):
    """[kv head][token][H] of the first tokens of sequence b; NaN where its page is none."""
    pages, heads, rows, H = values.shape
    out = torch.full((heads, tokens, H), math.nan, dtype=torch.float64)
    for t in range(tokens):
        page = int(table[b, t // rows])
        if 0 <= page < pages:
            out[:, t] = values[page, :, t % rows]
    return out


def ancestors(parents):
    """Of each row of one sequence the set of rows that it sees; None: no token."""
    seen = []
    for i, p in enumerate(parents):
        ok = -1 <= p < i and (p < 0 or seen[p] is not None)
        seen.append(((seen[p] if p >= 0 else set()) | {i}) if ok else None)
    return seen


def mask_words(seen, words):
    """The sets as 64-bit words, as torch holds them."""
    bits = [sum(1 << j for j in s or ()) for s in seen]
    return [[(w >> (64 * k) & (2 ** 64 - 1)) - ((w >> (64 * k + 63) & 1) << 64) for k in range(words)] for w in bits]


def attention(Q, values, table, lens, K=None, V=None, masks=None, scale=1.0):
    """N, m, l (numbers relative to m), and for the bounds A = sum p |v| and the largest sum |q| |k| of a row, all [b][head][row](..)."""
    n, heads, rows, H = Q.shape
    group = heads // values[0].shape[1]
    room = table.shape[1] * values[0].shape[2]
    N, A = torch.zeros(n, heads, rows, H, dtype=torch.float64), torch.zeros(n, heads, rows, H, dtype=torch.float64)
    m, l, size = torch.full((n, heads, rows), -math.inf, dtype=torch.float64), *torch.zeros(2, n, heads, rows, dtype=torch.float64)
    for b in range(n):
        tokens = min(max(int(lens[b]), 0), room)
        k, v = (sequence(x, table, b, tokens) for x in values)
        there = [int(table[b, t // values[0].shape[2]]) in range(values[0].shape[0]) for t in range(tokens)]
        for i in range(rows):
            drafted = []
            if masks is not None:
                words = [int(w) & (2 ** 64 - 1) for w in masks[b, i]]
                if not words[i // 64] >> (i % 64) & 1:
                    continue
                drafted = [j for j in range(rows) if words[j // 64] >> (j % 64) & 1]
            else:
                drafted = list(range(i + 1))
            at = [t for t in range(tokens) if there[t]]
            for h in range(heads):
                keys, vals = k[h // group][at], v[h // group][at]
                if K is not None:
                    keys = torch.cat([keys, K[b, h // group][drafted].double().cpu()])
                    vals = torch.cat([vals, V[b, h // group][drafted].double().cpu()])
                if not len(keys):
                    continue
                q = Q[b, h, i].double().cpu()
                s = (keys @ q) * scale
                m[b, h, i] = s.max()
                p = torch.exp(s - m[b, h, i])
                l[b, h, i] = p.sum()
                N[b, h, i] = (p.unsqueeze(1) * vals).sum(0)
                A[b, h, i] = (p.unsqueeze(1) * vals.abs()).sum(0)
                size[b, h, i] = (keys.abs() @ q.abs()).max() * scale
    return N, m, l, A, size


def bounds(N, m, l, A, size, H, keys, coarse=False):
    """How far (N, l relative to the kernel's own m), m and lse may be, and O in bf16.  fp32: H products of a score and their sum, then its
    product with scale log2(e) and the reference taken off (4 more), each 2^-24 of sum |q k| or less: ds.  An exponential: that, and an ulp of
    2^x.  P as two bf16 numbers: 2^-16.  Sums of `keys` terms in any order, four partial ones: (keys + 8) 2^-24; merges rescale a few
    times: 2^-20 covers them.  coarse: P of O as one bf16 number, each at most half a step off, 2^-8: of the sum of the |p v| that is as much."""
    ds = (H + 8) * 2.0 ** -24 * size
    rel = 2 * ds + 2.0 ** -16 + (keys + 8) * 2.0 ** -24 + 2.0 ** -20
    some = l > 0
    l1 = torch.where(some, l, torch.ones_like(l))
    O, a = N / l1.unsqueeze(-1), A / l1.unsqueeze(-1)
    return {"O": (2.0 ** -8) * O.abs() + (rel.unsqueeze(-1) * 2 + (2.0 ** -8 if coarse else 0)) * a, "N": rel.unsqueeze(-1) * A, "l": rel * l,
            "m": ds + 2.0 ** -22 * m.abs().nan_to_num(0, 0, 0), "lse": rel + ds + 2.0 ** -21 * m.abs().nan_to_num(0, 0, 0) + 2.0 ** -22}


def new_cache(gen, a2d, fmt, pages, kv_heads, page_rows, H, sigma=1.0):
    """A cache full of tokens (codes and scales drawn, not written by the library)."""
    K, V = (sigma * torch.randn(pages, kv_heads, page_rows, H, generator=gen) for _ in range(2))
    if fmt == "bf16":
        return K.bfloat16().cuda(), V.bfloat16().cuda()
    out = []
    for x in (K, V):
        codes, e = quantised(x, fmt)
        if fmt == "e4m3":
            c = codes.to(torch.uint8).view(torch.float8_e4m3fn)
        else:
            c = (codes[..., 0::2] + 16 * codes[..., 1::2]).to(torch.uint8)
        s = torch.full((*e.shape[:-1], 4), 127, dtype=torch.uint8)
        s[..., :e.shape[-1]] = (e + 127).to(torch.uint8)
        out.append((c.cuda(), s.cuda()))
    return out[0][0], out[1][0], out[0][1], out[1][1]
