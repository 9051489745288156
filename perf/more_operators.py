"""A paged cache of keys and values in 8 or 4 bits - written, read back - and the attention of a tree of drafted tokens
over it, as measurable cases.

`listed()` gives the fixed cases, `draw(rng)` one more of the same ranges, `prepare(case, seed)` what a program holds before
the call, `run(state)` one pass - in elementary torch operations, or with `own` through the public entry points of
`paper_2503_15758_amd.binding` -, `work(case)` the bytes and operations that a pass cannot do without and `exact(case, seed)`
its results in 64 bits.

Kinds of cases (key "op"):
  write   new rows of K and V into the pages of a batch's sequences.  "starts": the tokens that they begin at, "keep": of the
          drafted rows those that were accepted (an index), else all.  Codes and scales of the whole cache come out; "back": the
          sequences' tokens up to the last written one, read back, instead
  read    K and V of the tokens "first" .. "first" + "rows" - 1 of each sequence, in the model's type
  tree    from the parents of drafted tokens the bits of what each of them sees, and their positions
  attend  the drafted rows (their own K and V beside them) against caches of the lengths "lens": O in the model's type and lse, or
          with "partial" the unnormalised fp32 partial.  "tree": a tree of tokens, else a chain
A cache is pages [pages][kv head][page row][H] and a table [sequence][page]; "e4m3": a code of 8 bits for each value, "e2m1" of 4,
and a power of two (its exponent, a byte) for each 32 values of a row; "bf16": the values themselves.
"packed": Q, K and V are views of the [sequence][row][heads][H] tensors that a model keeps.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEAD_SIZES = (64, 80, 96, 128)
FORMATS = ("bf16", "e4m3", "e2m1")
BLOCK = 32                       # values that share a scale
LOWEST = -100                    # the smallest exponent of a scale
# largest value: fraction of a power of two, exponent of that power; smallest normal's exponent; bits of the fraction
CODES = {"e4m3": (0.875, 9, -6, 3), "e2m1": (0.75, 3, 0, 1)}


def _case(name, op, fmt, kv_heads, hdim, page_rows, **more):
    c = {"name": name, "op": op, "format": fmt, "dtype": "bf16", "heads": kv_heads, "kv_heads": kv_heads, "hdim": hdim,
         "page_rows": page_rows, "lens": "0", "rows": 1, "first": 0, "keep": False, "back": False, "tree": False,
         "partial": False, "packed": False}
    c.update(more)
    return c


def _many(*runs):
    """"n x length" runs as one text of lengths."""
    return ",".join(str(v) for n, v in runs for _ in range(n))


def listed():
    return [
        # serving: one new token of each of 64 sequences goes into the cache; latency
        _case("write 64 sequences, a token", "write", "e4m3", 8, 128, 64, lens=_many((40, 700), (23, 1999), (1, 0)), packed=True),
        # a long prompt goes into the cache
        _case("write 8x16384 prompt", "write", "e4m3", 8, 128, 64, rows=16384, packed=True),
        # an fp32 model's accepted drafts, four bits, and the sequences read back
        _case("write 5x40 kept e2m1 x 80, back", "write", "e2m1", 12, 80, 48, rows=40, dtype="f32", keep=True, back=True,
              lens="0,777,4095,1,2500"),
        # the cached part of a prompt, for the tile calls that take the rest of it
        _case("read 8x16384", "read", "e4m3", 8, 128, 64, rows=16384, lens="16384"),
        # a window of three sequences, four bits, one of them ends inside it
        _case("read 3x2999 e2m1 x 96", "read", "e2m1", 4, 96, 16, rows=2999, first=1001, dtype="f32", lens="4000,2222,9000"),
        # a small tree of one sequence
        _case("tree 1x7", "tree", "bf16", 1, 64, 64, rows=7, tree=True, lens="300"),
        # large trees of a batch, padded to one size
        _case("tree 64x250", "tree", "bf16", 1, 64, 64, rows=250, tree=True, lens=_many((63, 5000), (1, 0))),
        # seven drafted tokens over a short text: latency
        _case("attend 1x7, 8/2 heads x 64, 300", "attend", "bf16", 2, 64, 64, heads=8, rows=7, tree=True, lens="300"),
        # serving without drafts: one token of each of 8 sequences, to 16384 tokens
        _case("attend 8 sequences, a token", "attend", "e4m3", 8, 128, 64, heads=32, packed=True,
              lens="16384,777,12000,1,9001,16383,4096,15000"),
        # one long sequence among many short ones, three drafted tokens, four bits
        _case("attend 32 sequences, one long, e2m1", "attend", "e2m1", 4, 128, 64, heads=32, rows=3, packed=True,
              lens=_many((1, 32768), (20, 200), (10, 1111), (1, 0))),
        # a device's share of one long text, as a partial that is merged with the others'; odd pages, a ragged tree
        _case("attend 1x25 partial, 12/4 x 80, 50001", "attend", "e4m3", 4, 80, 48, heads=12, rows=25, tree=True, partial=True,
              lens="50001"),
        # large trees over long texts: more operations than bytes
        _case("attend 8x64 tree, 32/8, to 16384", "attend", "e4m3", 8, 128, 64, heads=32, rows=64, tree=True, packed=True,
              lens="16384,16384,12000,16000,9001,16383,14096,15000"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "read", "tree", "attend", "attend", "attend"])
    hdim, page = rng.choice(HEAD_SIZES), rng.choice([16, 48, 64, 128, 272])
    fmt = rng.choice(FORMATS) if op == "attend" else rng.choice(FORMATS[1:])
    sequences = _log_int(rng, 1, 64)
    if op == "tree":
        c = _case("", op, "bf16", 1, 64, 64, rows=rng.randint(8, 256), tree=True,
                  lens=",".join(str(_log_int(rng, 1, 30000)) for _ in range(sequences)))
    elif op == "attend":
        kv, group = _log_int(rng, 1, 16), rng.choice([1, 1, 2, 4, 8])
        rows = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 2, 100)])
        while True:                                            # (below the largest listed ones)
            sequences, most = _log_int(rng, 1, 64), _log_int(rng, 16, 65536)
            if sequences * kv * most <= 4000000 and sequences * kv * group * rows * (most + rows) <= 2.0e8:
                break
        lens = [rng.choice([most, most, _log_int(rng, 1, most), _log_int(rng, 1, most), 0]) for _ in range(sequences)]
        c = _case("", op, fmt, kv, hdim, page, heads=kv * group, rows=rows, tree=rows > 1 and rng.random() < 0.7,
                  partial=rng.random() < 0.25, packed=rng.random() < 0.5, lens=",".join(map(str, lens)))
    else:
        kv = _log_int(rng, 1, 16)
        sequences = _log_int(rng, 1, 16)
        rows = _log_int(rng, 1, max(1, 100000 // (sequences * kv)))
        lens = [rng.choice([0, _log_int(rng, 1, 5000)]) for _ in range(sequences)]
        c = _case("", op, fmt, kv, hdim, page, rows=rows, packed=rng.random() < 0.5, dtype="f32" if rng.random() < 0.3 else "bf16",
                  lens=",".join(map(str, lens)))
        if op == "write":
            c["keep"], c["back"] = rng.random() < 0.3, fmt == "e2m1"
        else:
            lens[0] = max(lens[0], 1)
            c["lens"] = ",".join(map(str, lens))
            c["first"] = rng.choice([0, rng.randint(0, max(lens) - 1)])
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------- inputs

def _lens(c):
    return [int(v) for v in c["lens"].split(",")]


def _held(c):
    """Tokens that the pages of each sequence have room for."""
    return [n + (c["rows"] if c["op"] == "write" else 0) for n in _lens(c)]


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _values(gen, shape, spread=False):
    """N(0, 1); "spread": some columns are far larger than others, as those of keys are."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    if spread:
        x *= torch.exp2(2.0 * torch.randn(shape[-1], generator=gen, device="cuda").clamp(-2, 1))
    return x


def _batch(gen, c, heads, dtype, spread=False):
    """[sequence][head][row][H]"""
    b = len(_lens(c))
    if c["packed"]:
        return _values(gen, (b, c["rows"], heads, c["hdim"]), spread).to(dtype).permute(0, 2, 1, 3)
    return _values(gen, (b, heads, c["rows"], c["hdim"]), spread).to(dtype)


def _parents(c, gen):
    """Of each row a token before it (row 0 follows the text); some sequences of a batch have fewer tokens than rows (-2)."""
    b, n = len(_lens(c)), c["rows"]
    row = torch.arange(n, device="cuda", dtype=torch.float32)
    p = torch.floor(torch.rand(b, n, generator=gen, device="cuda").sqrt() * row).clamp(max=row - 1).int()
    p[:, 0] = -1
    if b > 1 and n > 1:
        p[1::3, n - (n + 3) // 4:] = -2
    return p


def prepare(case, seed):
    c, gen = case, _generator(seed)
    lens, held = _lens(c), _held(c)
    need = [-(-n // c["page_rows"]) for n in held]
    s = {"case": c, "lens": _int32(lens), "most": max(held)}
    if c["op"] == "tree":
        s["parents"] = _parents(c, gen)
        return s
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = table
    shape = (pages, c["kv_heads"], c["page_rows"], c["hdim"])
    dtype = DTYPES[c["dtype"]]
    if c["op"] == "write":
        s["K"], s["V"] = _batch(gen, c, c["kv_heads"], dtype, True), _batch(gen, c, c["kv_heads"], dtype)
        s["index"] = None
        if c["keep"]:                                           # (row 0 and about a third of the others, in order, then nothing)
            chosen = torch.rand(len(lens), c["rows"], generator=gen, device="cuda") < 0.35
            chosen[:, 0] = True
            row = torch.arange(c["rows"], device="cuda").expand_as(chosen)
            row = torch.where(chosen, row, c["rows"]).sort(1).values
            s["index"] = torch.where(row < c["rows"], row, -1).int()
        if c["back"]:
            kept = (s["index"] >= 0).sum(1) if c["keep"] else torch.full((len(lens),), c["rows"], device="cuda")
            s["now"] = (s["lens"] + kept).int()
        blank = torch.zeros(shape, device="cuda")
        s["cache"] = _coded(blank, blank, c["format"])
        return s
    s["cache"] = _coded(_values(gen, shape, True), _values(gen, shape), c["format"])
    if c["op"] == "attend":
        s["scale"] = 1.0 / math.sqrt(c["hdim"])
        s["Q"] = _batch(gen, c, c["heads"], dtype)
        s["K"], s["V"] = _batch(gen, c, c["kv_heads"], dtype, True), _batch(gen, c, c["kv_heads"], dtype)
        s["masks"] = _tree(_parents(c, gen), s["lens"])[0] if c["tree"] else None
    return s


# ------------------------------------------------------------------------------------- the plain forms

def _blocks(x):
    """[..][blocks][32], the last block of 16 with zeros behind."""
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))


def _quantised(x, fmt):
    """Codes of the values x [..][H] and their scales, four bytes a row."""
    fraction, power, lowest, bits = CODES[fmt]
    y = _blocks(x.float())
    m, e = torch.frexp(y.abs().amax(-1, keepdim=True))
    s = torch.where(m == 0, LOWEST, (e - power + (m > fraction)).clamp(min=LOWEST))
    y = torch.ldexp(y, -s)
    step = torch.exp2((torch.frexp(y.abs())[1] - 1).clamp(min=lowest).float() - bits)
    y = (torch.round(y / step) * step).flatten(-2)[..., :x.shape[-1]]
    scales = torch.nn.functional.pad(s.squeeze(-1) + 127, (0, 4 - s.shape[-2]), value=127).to(torch.uint8)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn), scales
    a = y.abs()
    code = sum((a >= v).int() for v in (0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)) + 8 * torch.signbit(y).int()
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), scales


def _coded(K, V, fmt):
    """The tensors of a cache that holds K and V."""
    if fmt == "bf16":
        return K.to(torch.bfloat16), V.to(torch.bfloat16)
    (k, ks), (v, vs) = _quantised(K, fmt), _quantised(V, fmt)
    return k, v, ks, vs


def _meant(codes, scales, fmt, hdim):
    """The values that codes stand for, fp32."""
    if fmt == "bf16":
        return codes.float()
    if fmt == "e2m1":
        worth = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
        worth = torch.cat([worth, -worth])
        y = torch.stack([worth[(codes & 15).int()], worth[(codes >> 4).int()]], -1).flatten(-2)
    else:
        y = codes.float()
    y = _blocks(y) * torch.exp2(scales[..., :-(-hdim // BLOCK), None].float() - 127)
    return y.flatten(-2)[..., :hdim]


def _bytes(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _tokens(c, cache, table, first, rows):
    """K and V, fp32 [sequence][kv head][row][H], of the tokens from `first` on."""
    t = first + torch.arange(rows, device="cuda")
    page = table[:, (t // c["page_rows"]).clamp(max=table.shape[1] - 1)].clamp(min=0).long()
    off = (t % c["page_rows"]).expand_as(page)
    got = []
    for i in range(2):
        codes = _bytes(cache[i])[page, :, off]
        scales = cache[2 + i][page, :, off] if c["format"] != "bf16" else None
        got.append(_meant(codes.view(cache[i].dtype), scales, c["format"], c["hdim"]).transpose(1, 2))
    return got


def _read(c, cache, table, lens, first, rows):
    behind = first + torch.arange(rows, device="cuda") >= lens.unsqueeze(1)
    return tuple(x.masked_fill(behind[:, None, :, None], 0).to(DTYPES[c["dtype"]]) for x in _tokens(c, cache, table, first, rows))


def _write(s):
    c = s["case"]
    b, n = len(_lens(c)), c["rows"]
    index = s["index"] if c["keep"] else torch.arange(n, device="cuda").expand(b, -1)
    t = s["lens"].unsqueeze(1) + torch.arange(n, device="cuda")
    page = s["table"].gather(1, (t // c["page_rows"]).clamp(max=s["table"].shape[1] - 1))
    written = (index >= 0) & (index < n)
    seq = torch.arange(b, device="cuda").unsqueeze(1).expand(-1, n)
    seq, row, page, off = seq[written], index[written].long(), page[written].long(), (t % c["page_rows"])[written]
    new = _coded(s["K"][seq, :, row], s["V"][seq, :, row], c["format"])
    for held, x in zip(s["cache"], new):
        _bytes(held)[page, :, off] = _bytes(x)


def _tree(parents, lens):
    """(bits [sequence][row][64-bit word] of the rows that a row sees, positions [sequence][1][row]); padding sees nothing."""
    b, n = parents.shape
    row = torch.arange(n, device="cuda")
    p = parents.long()
    # points 0: the text, 1 .. n: the rows, n + 1: no token (padding, and what follows it)
    up = torch.where((p >= -1) & (p < row), p + 1, n + 1)
    up = torch.nn.functional.pad(torch.nn.functional.pad(up, (1, 0)), (0, 1), value=n + 1)
    sees = torch.eye(n + 2, dtype=torch.bool, device="cuda").repeat(b, 1, 1)
    for _ in range(n.bit_length()):                            # (twice as far up each time)
        sees = sees | sees.gather(1, up.unsqueeze(2).expand_as(sees))
        up = up.gather(1, up)
    sees = sees[:, 1:n + 1]
    real = ~sees[..., n + 1]
    sees = sees[..., 1:n + 1] & real.unsqueeze(2)
    position = (lens.unsqueeze(1) + sees.sum(2) - 1).where(real, torch.zeros((), dtype=torch.int64, device="cuda"))
    words = -(-n // 64)
    bit = torch.nn.functional.pad(sees, (0, 64 * words - n)).unflatten(2, (words, 64)).long()
    return (bit << torch.arange(64, device="cuda")).sum(3), position.int().unsqueeze(1)


def _attend(s):
    c = s["case"]
    b, n, kv = len(_lens(c)), c["rows"], c["kv_heads"]
    K, V = _tokens(c, s["cache"], s["table"], 0, s["most"])
    K, V = torch.cat([K, s["K"].float()], 2), torch.cat([V, s["V"].float()], 2)
    row = torch.arange(n, device="cuda")
    if s["masks"] is not None:
        sees = ((s["masks"][:, :, row // 64] >> (row % 64)) & 1).bool()
        real = sees[:, row, row]
        sees = sees & real.unsqueeze(2)
    else:
        sees = (row <= row.unsqueeze(1)).expand(b, -1, -1)
        real = torch.ones(b, n, dtype=torch.bool, device="cuda")
    cached = (torch.arange(s["most"], device="cuda") < s["lens"].unsqueeze(1)).unsqueeze(1) & real.unsqueeze(2)
    hidden = ~torch.cat([cached, sees], 2)[:, None, None]
    x = torch.matmul(s["Q"].float().reshape(b, kv, -1, c["hdim"]), K.transpose(2, 3).contiguous()) * s["scale"]
    x = x.view(b, kv, -1, n, x.shape[-1]).masked_fill_(hidden, -math.inf).flatten(2, 3)
    m = x.amax(3, keepdim=True)
    p = torch.exp(x - m.where(m > -math.inf, torch.zeros_like(m)))
    l = p.sum(3, keepdim=True)
    N = torch.matmul(p, V.contiguous())
    shape = (b, c["heads"], n)
    if c["partial"]:
        return {"O_part": N.view(*shape, -1), "m": m.view(shape), "l": l.view(shape)}
    O = torch.where(l > 0, N / l, torch.zeros_like(N))
    return {"O": O.view(*shape, -1).to(s["Q"].dtype), "lse": (m + torch.log(l)).view(shape)}


# --------------------------------------------------------------------------------------------- a pass

def run(s):
    c = s["case"]
    if own:
        from paper_2503_15758_amd import binding as a2d
        if c["op"] == "tree":
            masks, positions = a2d.tree_masks(s["parents"], s["lens"])
            return {"masks": masks, "positions": positions}
        dtype = DTYPES[c["dtype"]]
        if c["op"] == "read":
            K, V = a2d.cache_read(s["cache"], s["table"], s["lens"], c["rows"], first=c["first"], out_dtype=dtype)
            return {"K": K, "V": V}
        if c["op"] == "write":
            a2d.cache_write(s["cache"], s["table"], s["K"], s["V"], s["lens"], index=s["index"])
            if c["back"]:
                K, V = a2d.cache_read(s["cache"], s["table"], s["now"], s["most"], out_dtype=dtype)
                return {"K": K, "V": V}
            return _whole(s)
        out = a2d.partial_fwd_cached(s["Q"], s["cache"], s["table"], s["lens"], K=s["K"], V=s["V"], masks=s["masks"],
                                     scale=s["scale"], max_tokens=s["most"], normalised=not c["partial"])
        return dict(zip(("O_part", "m", "l") if c["partial"] else ("O", "lse"), out))
    if c["op"] == "tree":
        masks, positions = _tree(s["parents"], s["lens"])
        return {"masks": masks, "positions": positions}
    if c["op"] == "read":
        K, V = _read(c, s["cache"], s["table"], s["lens"], c["first"], c["rows"])
        return {"K": K, "V": V}
    if c["op"] == "write":
        _write(s)
        if c["back"]:
            K, V = _read(c, s["cache"], s["table"], s["now"], 0, s["most"])
            return {"K": K, "V": V}
        return _whole(s)
    return _attend(s)


def _whole(s):
    """The cache's tensors: codes, and scales as the powers of two that they are."""
    named = dict(zip(("K", "V", "K_scales", "V_scales"), s["cache"]))
    return {k: x.view(torch.float8_e8m0fnu) if x.dtype == torch.uint8 else x for k, x in named.items()}


# --------------------------------------------------------------------------- what a pass cannot do without

def _row_bytes(c):
    """K and V of a token of one head in the cache."""
    H = c["hdim"]
    if c["format"] == "bf16":
        return 4 * H
    return 2 * (H if c["format"] == "e4m3" else H // 2) + 2 * -(-H // BLOCK)


def work(case):
    c, lens = case, _lens(case)
    e, H, b = (2 if c["dtype"] == "bf16" else 4), c["hdim"], len(lens)
    if c["op"] == "tree":
        return {"bytes": b * c["rows"] * (8 + 8 * -(-c["rows"] // 64)), "flops": 0}
    if c["op"] == "write":
        rows = b * c["kv_heads"] * c["rows"]
        if c["keep"]:
            rows = 35 * rows // 100
        n = rows * (2 * H * e + _row_bytes(c))
        if c["back"]:
            held = sum(v + rows // (b * c["kv_heads"]) for v in lens) * c["kv_heads"]
            n += held * _row_bytes(c) + b * c["kv_heads"] * max(_held(c)) * 2 * H * e
        return {"bytes": n, "flops": 0}
    if c["op"] == "read":
        held = sum(min(c["rows"], max(0, v - c["first"])) for v in lens) * c["kv_heads"]
        return {"bytes": held * _row_bytes(c) + b * c["kv_heads"] * c["rows"] * 2 * H * e, "flops": 0}
    q = b * c["heads"] * c["rows"]
    written = 4 * H + 8 if c["partial"] else 2 * H + 4
    n = sum(lens) * c["kv_heads"] * _row_bytes(c) + b * c["kv_heads"] * c["rows"] * 4 * H + q * (2 * H + written)
    # (of the drafted tokens a row sees half, at the most)
    scores = c["heads"] * c["rows"] * (sum(lens) + b * (c["rows"] + 1) // 2)
    return {"bytes": n, "flops": 4 * scores * H}


# ------------------------------------------------------------------------------------------- in 64 bits

def _worth(fmt):
    """The values of the codes without a sign, rising."""
    if fmt == "e2m1":
        return [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]


def _nearest(x, fmt):
    """(code values with their signs, exponents of the scales) of x [..][H], by search among all codes."""
    worth = torch.tensor(_worth(fmt), dtype=torch.float64, device="cuda")
    H = x.shape[-1]
    values, exponents = torch.empty(x.shape, dtype=torch.float64, device="cuda"), []
    for first in range(0, H, BLOCK):
        y = x[..., first:first + BLOCK].double()
        top = y.abs().amax(-1, keepdim=True)
        s = torch.ceil(torch.log2(top / worth[-1])).clamp(min=LOWEST)
        s = torch.where(top > worth[-1] * torch.exp2(s), s + 1, s)                     # (a logarithm that was rounded)
        s = torch.where((s > LOWEST) & (top <= worth[-1] * torch.exp2(s - 1)), s - 1, s)
        y = y / torch.exp2(s)
        above = torch.searchsorted(worth, y.abs().contiguous()).clamp(1, worth.numel() - 1)
        up, down = worth[above] - y.abs(), y.abs() - worth[above - 1]
        code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, above - 1)
        values[..., first:first + BLOCK] = torch.copysign(worth[code], y)
        exponents.append(s)
    return values, torch.cat(exponents, -1)


def _decoded(c, cache, i):
    """All pages' K (i = 0) or V in 64 bits."""
    if c["format"] == "bf16":
        return cache[i].double()
    if c["format"] == "e4m3":
        x = cache[i].double()
    else:
        worth = torch.tensor(_worth("e2m1"), dtype=torch.float64, device="cuda")
        x = torch.empty(*cache[i].shape[:-1], c["hdim"], dtype=torch.float64, device="cuda")
        for half in range(2):
            code = ((cache[i] >> (4 * half)) & 15).long()
            x[..., half::2] = worth[code & 7] * torch.where(code > 7, -1.0, 1.0)
    for block in range(-(-c["hdim"] // BLOCK)):
        x[..., block * BLOCK:(block + 1) * BLOCK] *= torch.exp2(cache[2 + i][..., block:block + 1].double() - 127)
    return x


def _sequence(c, s, pages, b, tokens):
    """[kv head][token][H] of sequence b from its decoded pages."""
    n = -(-tokens // c["page_rows"])
    x = pages[s["table"][b, :n].long()].transpose(0, 1).reshape(c["kv_heads"], -1, c["hdim"])
    return x[:, :tokens]


def _sees(parents):
    """[row][row] of one sequence, on the host; rows that are padding see nothing."""
    seen = []
    for i, p in enumerate(parents):
        if p < -1 or p >= i or (p >= 0 and seen[p] is None):
            seen.append(None)
        else:
            seen.append((seen[p] if p >= 0 else frozenset()) | {i})
    return seen


def exact(case, seed):
    c, s = case, prepare(case, seed)
    lens = _lens(c)
    if c["op"] == "tree":
        words = -(-c["rows"] // 64)
        masks, positions = [], []
        for b, p in enumerate(s["parents"].tolist()):
            seen = _sees(p)
            bits = [sum(1 << j for j in v or ()) for v in seen]
            masks.append([[(w >> (64 * k) & (2 ** 64 - 1)) - ((w >> (64 * k + 63) & 1) << 64) for k in range(words)] for w in bits])
            positions.append([[lens[b] + len(v) - 1 if v else 0 for v in seen]])
        return {"masks": torch.tensor(masks), "positions": _int32(positions)}
    if c["op"] == "write":
        if s["K"].numel() > 3e7:
            return None
        out = {}
        for i, name in enumerate(("K", "V")):
            pages = _decoded(c, s["cache"], i) * 0
            values, exponents = _nearest(s[name], c["format"])
            powers = torch.ones(*pages.shape[:3], 4, dtype=torch.float64, device="cuda")
            if not c["back"]:
                powers[..., :exponents.shape[-1]] = 2.0 ** LOWEST
            for b, n in enumerate(lens):
                rows = [r for r in s["index"][b].tolist() if r >= 0] if c["keep"] else list(range(c["rows"]))
                t = torch.arange(n, n + len(rows), device="cuda")
                page, off = s["table"][b][t // c["page_rows"]].long(), t % c["page_rows"]
                pages[page, :, off] = values[b, :, rows].transpose(0, 1)
                e = torch.exp2(exponents[b, :, rows]).transpose(0, 1)
                for k in range(e.shape[-1]):
                    powers[page, :, off, k] = e[..., k]
            if c["back"]:
                powers = powers[..., :exponents.shape[-1]].repeat_interleave(BLOCK, -1)[..., :c["hdim"]]
                back = torch.zeros(len(lens), c["kv_heads"], s["most"], c["hdim"], dtype=torch.float64, device="cuda")
                for b, n in enumerate(s["now"].tolist()):
                    back[b, :, :n] = _sequence(c, s, pages * powers, b, n)
                out[name] = back
            else:
                out[name], out[name + "_scales"] = pages, powers
        return out
    pages = [_decoded(c, s["cache"], i) for i in range(2)]
    if c["op"] == "read":
        out = {}
        for i, name in enumerate(("K", "V")):
            x = torch.zeros(len(lens), c["kv_heads"], c["rows"], c["hdim"], dtype=torch.float64, device="cuda")
            for b, n in enumerate(lens):
                end = min(n, c["first"] + c["rows"])
                if end > c["first"]:
                    x[b, :, :end - c["first"]] = _sequence(c, s, pages[i], b, end)[:, c["first"]:]
            out[name] = x
        return out
    b, n, group = len(lens), c["rows"], c["heads"] // c["kv_heads"]
    shape = (b, c["heads"], n)
    N = torch.zeros(*shape, c["hdim"], dtype=torch.float64, device="cuda")
    m, l = torch.full(shape, -math.inf, dtype=torch.float64, device="cuda"), torch.zeros(shape, dtype=torch.float64, device="cuda")
    masks = s["masks"].tolist() if c["tree"] else None
    for q, tokens in enumerate(lens):
        sees = torch.zeros(n, n, dtype=torch.bool)
        for i in range(n):
            for j in range(n):
                sees[i, j] = j <= i if masks is None else bool(masks[q][i][j // 64] >> (j % 64) & 1)
        sees = sees.cuda()
        K, V = (torch.cat([_sequence(c, s, x, q, tokens), s[name][q].double()], 1) for x, name in zip(pages, ("K", "V")))
        see = torch.cat([sees.diagonal().unsqueeze(1).expand(-1, tokens), sees & sees.diagonal().unsqueeze(1)], 1)
        for h in range(c["heads"]):
            a = (s["Q"][q, h].double() @ K[h // group].t().contiguous()) * s["scale"]
            a = a.masked_fill(~see, -math.inf)
            m[q, h] = a.amax(1)
            w = (a - m[q, h].unsqueeze(1)).exp().nan_to_num(0.0)
            l[q, h] = w.sum(1)
            N[q, h] = w @ V[h // group]
    if c["partial"]:
        return {"O_part": N, "m": m, "l": l}
    return {"O": torch.where(l.unsqueeze(3) > 0, N / l.unsqueeze(3), 0.0), "lse": m + torch.log(l)}
