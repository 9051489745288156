"""Attention with rules on its scores (a tanh cap, a bias that falls with distance, documents, prefixes) and rotary
positions with several axes, as measurable cases.

`listed()` gives the fixed cases, `draw(rng)` one more of the same ranges, `prepare(case, seed)` what a program holds before
the call, `run(state)` one pass - in elementary torch operations, or with `own` through the public entry points of
`paper_2503_15758_amd.binding` -, `work(case)` the bytes and operations that a pass cannot do without and `exact(case, seed)`
its results in 64 bits.

Kinds of cases (key "op"):
  fwd     a query block against a key/value block: O in the inputs' type and lse.  With "docs" the masks of the packed
          documents are built from their boundaries in the pass
  bwd     the gradients of such a block, in the inputs' type, from the saved O and lse
  rotary  Q and K turned by the positions of their tokens; "inverse": the gradients of both turned back, fp32 sums in
          and the model's type out
"docs": "first token:prefix length, .." of the documents of a packed sequence, "end" the token behind the last one (tokens
from there on are padding, which sees nothing).  "lens": the lengths of the sequences of a batch, one token of each of which
asks (their heads follow one another).  "step": tokens between rows, as in a cyclic layout.  "packed": Q, K, V, O, dO are
views of the [rows][heads][H] tensors that a model keeps.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEAD_SIZES = (64, 80, 96, 128)


def _tile(name, op, heads, kv_heads, nq, nkv, hdim, **more):
    c = {"name": name, "op": op, "dtype": "bf16", "heads": heads, "kv_heads": kv_heads, "nq": nq, "nkv": nkv, "hdim": hdim,
         "q_off": 0, "kv_off": 0, "step": 1, "causal": False, "cap": 0.0, "slopes": False, "docs": "", "end": 0, "lens": "",
         "sigma": 1.0, "packed": False}
    c.update(more)
    return c


def _turn(name, heads, kv_heads, rows, hdim, **more):
    c = {"name": name, "op": "rotary", "dtype": "bf16", "heads": heads, "kv_heads": kv_heads, "sets": 1, "rows": rows,
         "hdim": hdim, "sections": "16,24,24", "interleaved": False, "inverse": False, "far": 0, "packed": False}
    c.update(more)
    return c


def listed():
    return [
        # one new token of each of 8 sequences, grouped heads: latency
        _turn("rotary 8 sequences, a token", 256, 64, 1, 128, sets=8, far=100000),
        # a video's tokens (time, height, width), Q and K read where a packed projection left them
        _turn("rotary 32/8 x 16384 video", 32, 8, 16384, 128, packed=True),
        # the gradients of Q and K of an image's tokens on the way back, fp32 sums of a ragged tile
        _turn("rotary back 24 x 2999 x 80", 24, 24, 2999, 80, sections="20,20", interleaved=True, inverse=True),
        # the smallest tile of an fp32 model: 128 rows of a 256-token sequence on a 2 x 2 grid, a distance bias
        _tile("fwd fp32 2x128x128 bias", "fwd", 2, 2, 128, 128, 64, dtype="f32", q_off=128, slopes=True, causal=True),
        # a training tile of a model with capped scores and grouped heads: the diagonal block of its sequence
        _tile("fwd 32/8x4096 capped", "fwd", 32, 8, 4096, 4096, 128, causal=True, cap=30.0, sigma=3.0),
        # packed documents, instructions read both ways (prefixes), a distance bias, padding behind
        _tile("fwd 16x8192 documents bias", "fwd", 16, 16, 8192, 8192, 64, slopes=True,
              docs="0:200,1500:0,1517:900,4100:64,4101:0,4800:512", end=8000),
        # serving: one token of each of 8 sequences against caches of up to 16384 tokens, capped
        _tile("fwd 8 sequences, a token", "fwd", 256, 64, 1, 16384, 128, cap=30.0, sigma=3.0,
              lens="16384,777,12000,1,9001,16383,4096,15000"),
        # long-context prefill: capped, a distance bias, one long document behind a short one
        _tile("fwd 8x16384 long", "fwd", 8, 8, 16384, 16384, 128, cap=50.0, slopes=True, sigma=3.0, docs="0:0,1999:100",
              end=16384),
        # the gradients of the capped training tile
        _tile("bwd 32/8x4096 capped", "bwd", 32, 8, 4096, 4096, 128, causal=True, cap=30.0, sigma=3.0),
        # and of packed documents of a model with 80-wide heads, activations read in place
        _tile("bwd 12/4x2999 documents", "bwd", 12, 4, 2999, 2999, 80, slopes=True, packed=True,
              docs="0:50,333:0,1024:400,2500:1", end=2900),
        # fp32 gradients of a ragged tile, capped, biased, the mask's diagonal through it
        _tile("bwd fp32 8x700x900", "bwd", 8, 8, 700, 900, 96, dtype="f32", causal=True, q_off=300, kv_off=100, cap=20.0,
              slopes=True, sigma=2.0),
        # documents alone: the gradients of a long packed sequence
        _tile("bwd 16x8192 documents", "bwd", 16, 16, 8192, 8192, 128, docs="0:0,2048:0,3000:0,7000:0", end=8192),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (below the largest listed ones)
_MOST_SCORES = {("bf16", "fwd"): 1.0e9, ("bf16", "bwd"): 5.0e8, ("f32", "fwd"): 2.0e7, ("f32", "bwd"): 5.0e6}


def _draw_docs(rng, c):
    n = rng.randint(1, 12)
    first, last = c["kv_off"], c["kv_off"] + c["nkv"] * c["step"]
    starts = sorted({first} | {rng.randint(first, last - 1) for _ in range(n - 1)})
    c["docs"] = ",".join("%d:%d" % (s, rng.choice([0, 0, rng.randint(1, max(1, c["nkv"] // 2))])) for s in starts)
    c["end"] = rng.choice([last, last - rng.randint(0, max(0, last - starts[-1] - 1))])
    c["causal"] = False


def draw(rng):
    op = rng.choice(["rotary", "fwd", "fwd", "bwd", "bwd", "token"])
    hdim = rng.choice(HEAD_SIZES)
    group = rng.choice([1, 1, 2, 4, 8])
    if op == "rotary":
        kv = _log_int(rng, 1, 16)
        half = hdim // 2
        cuts = sorted(rng.randint(1, half) for _ in range(rng.randint(0, 2)))
        sections = [b - a for a, b in zip([0] + cuts, cuts + [rng.choice([half, half, max(cuts + [1])])]) if b > a]
        sets = rng.choice([1, 1, 2, 5])
        rows = _log_int(rng, 1, max(1, 500000 // (kv * group * sets)))
        c = _turn("", sets * kv * group, sets * kv, rows, hdim, sets=sets, sections=",".join(map(str, sections)),
                  interleaved=rng.random() < 0.5, inverse=rng.random() < 0.4, far=rng.choice([0, 0, 1000000]),
                  packed=rng.random() < 0.4, dtype="f32" if rng.random() < 0.2 else "bf16")
        del c["name"]
        return c
    fp32 = op != "token" and rng.random() < 0.25
    if op == "token":
        seqs, kv = rng.randint(1, 12), _log_int(rng, 1, 8)
        nkv = _log_int(rng, 64, 16384)
        c = _tile("", "fwd", seqs * kv * group, seqs * kv, rng.choice([1, 1, 1, 2, 5]), nkv, hdim,
                  lens=",".join(str(rng.choice([nkv, _log_int(rng, 1, nkv)])) for _ in range(seqs)))
    else:
        kv = _log_int(rng, 1, 8)
        lo, hi = (64, 1024) if fp32 else (128, 16384)
        while True:
            nq, nkv = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
            if kv * group * nq * nkv <= _MOST_SCORES["f32" if fp32 else "bf16", op]:
                break
        c = _tile("", op, kv * group, kv, nq, nkv, hdim, dtype="f32" if fp32 else "bf16", packed=rng.random() < 0.25,
                  step=rng.choice([1, 1, 1, 4]))
        mask = rng.choice(["causal", "docs", "docs", "none"])
        c["kv_off"] = rng.choice([0, 0, 100])
        c["q_off"] = c["kv_off"] + rng.choice([0, 0, rng.randint(0, c["nkv"])]) * c["step"]
        if c["step"] > 1:
            c["q_off"] += rng.randint(0, 3)
        if mask == "causal":
            c["causal"] = True
        elif mask == "docs":
            _draw_docs(rng, c)
    c["cap"] = rng.choice([0.0, 0.0, 20.0, 30.0, 50.0])
    c["slopes"] = rng.random() < 0.4
    c["sigma"] = 3.0 if c["cap"] else 1.0
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, shape, dtype, sigma=1.0):
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return (x * sigma if sigma != 1.0 else x).to(dtype)


def _heads_tensor(gen, heads, rows, hdim, dtype, packed, sigma=1.0):
    """[heads][rows][H]; packed: a view of a [rows][heads][H] tensor."""
    if packed:
        return _normal(gen, (rows, heads, hdim), dtype, sigma).permute(1, 0, 2)
    return _normal(gen, (heads, rows, hdim), dtype, sigma)


def _documents(c):
    """(first tokens, end; prefix lengths) as lists."""
    docs = [tuple(int(v) for v in d.split(":")) for d in c["docs"].split(",")]
    return [d[0] for d in docs] + [c["end"]], [d[1] for d in docs]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _document_ranges(c, starts, prefix):
    """The tokens that each query row may see: of its own document up to itself, or its prefix; none of padding."""
    token = c["q_off"] + torch.arange(c["nq"], device="cuda", dtype=torch.int32) * c["step"]
    d = (token.unsqueeze(1) >= starts.unsqueeze(0)).sum(1) - 1
    inside = (d >= 0) & (d < prefix.numel())
    d = d.clamp(0, prefix.numel() - 1)
    first, last = starts[d], starts[d + 1]
    end = torch.minimum(last, torch.maximum(token + 1, first + prefix[d]))
    both = torch.stack([first, end], 1)
    return torch.where(inside.unsqueeze(1), both, torch.zeros_like(both))


def _length_ranges(c):
    """[sequence][row]: sequence b has the first lens[b] tokens of its cache."""
    lens = _int32([int(v) for v in c["lens"].split(",")])
    end = lens.unsqueeze(1).expand(-1, c["nq"])
    return torch.stack([torch.zeros_like(end), end], 2).contiguous()


def _slopes(c):
    h = c["heads"]
    return torch.exp2(-8.0 * torch.arange(1, h + 1, device="cuda", dtype=torch.float32) / h)


def _positions(c, gen):
    """[axis][row], or [set][axis][row]: time, height and width of a video of frames of 24 x 40 tokens that starts at
    some time; with "far" every axis of every set anywhere up to there."""
    axes, rows, sets = len(c["sections"].split(",")), c["rows"], c["sets"]
    if c["far"] or sets > 1:
        p = torch.randint(0, max(c["far"], rows + 1), (sets, axes, rows), generator=gen, device="cuda", dtype=torch.int32)
    else:
        t = torch.arange(rows, device="cuda", dtype=torch.int32)
        p = torch.stack([17 + t // 960, t // 40 % 24, t % 40][:axes]).unsqueeze(0)
    return p.contiguous() if sets > 1 else p[0].contiguous()


def _frequencies(c):
    """(radians a position, axis) of each pair of columns, on the host: one falling sequence over the pairs of all axes."""
    sections = [int(v) for v in c["sections"].split(",")]
    pairs = sum(sections)
    freqs = torch.tensor([10000.0 ** (-2.0 * p / c["hdim"]) for p in range(pairs)], dtype=torch.float64)
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], dtype=torch.uint8)
    return freqs, axis


def prepare(case, seed):
    c, gen = case, _generator(seed)
    dtype, H = DTYPES[c["dtype"]], c["hdim"]
    s = {"case": c}
    if c["op"] == "rotary":
        given = torch.float32 if c["inverse"] else dtype        # (gradients arrive as the fp32 sums of a tile)
        s["Q"] = _heads_tensor(gen, c["heads"], c["rows"], H, given, c["packed"] and not c["inverse"])
        s["K"] = _heads_tensor(gen, c["kv_heads"], c["rows"], H, given, c["packed"] and not c["inverse"])
        s["positions"] = _positions(c, gen)
        s["freqs"], s["axis"] = _frequencies(c)
        s["freqs_device"], s["axis_device"] = s["freqs"].cuda(), s["axis"].cuda()
        return s
    s["scale"] = 1.0 / math.sqrt(H)
    s["Q"] = _heads_tensor(gen, c["heads"], c["nq"], H, dtype, c["packed"], c["sigma"])
    s["K"] = _heads_tensor(gen, c["kv_heads"], c["nkv"], H, dtype, c["packed"])
    s["V"] = _heads_tensor(gen, c["kv_heads"], c["nkv"], H, dtype, c["packed"])
    s["slopes"] = _slopes(c) if c["slopes"] else None
    s["ranges"] = None
    if c["docs"]:
        starts, prefix = _documents(c)
        s["starts"], s["prefix"] = _int32(starts), _int32(prefix)
        if c["op"] == "bwd":                                    # (kept from the forward)
            s["ranges"] = _document_ranges(c, s["starts"], s["prefix"])
    elif c["lens"]:
        s["ranges"] = _length_ranges(c)
    if c["op"] == "bwd":
        s["dO"] = _heads_tensor(gen, c["heads"], c["nq"], H, dtype, c["packed"])
        O, s["lse"] = _attention(s, s["ranges"])
        s["O"] = torch.empty_like(s["dO"])                      # (keeps the strides of a packed dO)
        s["O"].copy_(O)
    return s


# ------------------------------------------------------------------------------------- the plain forms

def _hidden(c, ranges):
    """[1 or sequences][1][row][key]: the scores that are masked, or None."""
    i = c["q_off"] + torch.arange(c["nq"], device="cuda", dtype=torch.int64).unsqueeze(1) * c["step"]
    u = c["kv_off"] + torch.arange(c["nkv"], device="cuda", dtype=torch.int64).unsqueeze(0) * c["step"]
    h = None
    if c["causal"]:
        h = (i < u)[None, None]
    if ranges is not None:
        r = ranges.view(-1, 1, c["nq"], 1, 2)
        out = (u < r[..., 0]) | (u >= r[..., 1])
        h = out if h is None else h | out
    return h


def _by_head(c, x, sequences):
    """[heads][nq][..] <-> [sequences][heads of one][nq][..] (a view)"""
    return x.view(sequences, c["heads"] // sequences, *x.shape[1:])


def _scores(s, Q, K, ranges):
    """The scores [heads][nq][nkv] in fp32 with -inf where they are masked; the tanh of the cap beside them, or None."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    kt = K.transpose(1, 2).contiguous()
    x = torch.bmm(Q.reshape(c["kv_heads"], group * c["nq"], c["hdim"]), kt).view(c["heads"], c["nq"], c["nkv"]) * s["scale"]
    t = None
    if c["cap"]:
        t = torch.tanh(x / c["cap"])
        x = t * c["cap"]
    if s["slopes"] is not None:
        i = c["q_off"] - c["kv_off"] + torch.arange(c["nq"], device="cuda").unsqueeze(1) * c["step"]
        far = (i - torch.arange(c["nkv"], device="cuda").unsqueeze(0) * c["step"]).abs().float()
        x = x - s["slopes"].view(-1, 1, 1) * far
    hidden = _hidden(c, ranges)
    if hidden is not None:
        _by_head(c, x, hidden.shape[0]).masked_fill_(hidden, -math.inf)
    return x, t


def _attention(s, ranges):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    x, _ = _scores(s, s["Q"].float(), s["K"].float(), ranges)
    m = x.amax(2, keepdim=True)
    m0 = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(x - m0)
    l = p.sum(2, keepdim=True)
    n = torch.bmm(p.view(c["kv_heads"], group * c["nq"], c["nkv"]), s["V"].float().contiguous()).view(c["heads"], c["nq"], -1)
    some = l > 0
    O = torch.where(some, n / torch.where(some, l, torch.ones_like(l)), torch.zeros_like(n))
    lse = torch.where(some, m0 + torch.log(l), torch.full_like(l, -math.inf))
    return O.to(s["Q"].dtype), lse.squeeze(2)


def _gradients(s):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    rows = (c["kv_heads"], group * c["nq"])
    Q, K, V = s["Q"].float(), s["K"].float().contiguous(), s["V"].float()
    dO = s["dO"].float()
    x, t = _scores(s, Q, K, s["ranges"])
    lse = s["lse"].unsqueeze(2)
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse))
    delta = (dO * s["O"].float()).sum(2, keepdim=True)
    dp = torch.bmm(dO.reshape(*rows, -1), V.transpose(1, 2).contiguous()).view(x.shape)
    dz = p * (dp - delta)
    if t is not None:
        dz = dz * (1.0 - t * t)
    dz = dz.view(*rows, c["nkv"]) * s["scale"]
    dQ = torch.bmm(dz, K).view(c["heads"], c["nq"], -1)
    dK = torch.bmm(dz.transpose(1, 2).contiguous(), Q.reshape(*rows, -1))
    dV = torch.bmm(p.view(*rows, c["nkv"]).transpose(1, 2).contiguous(), dO.reshape(*rows, -1))
    return tuple(g.to(s["Q"].dtype) for g in (dQ, dK, dV))


def _rotated(s, x):
    c = s["case"]
    pos = s["positions"].view(c["sets"], -1, 1, c["rows"]).double()                   # [set][axis][1][row]
    angle = pos[:, s["axis_device"].long()] * s["freqs_device"].view(1, -1, 1, 1)     # [set][pair][1][row]: far positions
    angle = angle.permute(0, 2, 3, 1)                                                 # [set][1][row][pair]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["inverse"]:
        sin = -sin
    pairs = s["freqs"].numel()
    y = x.float().reshape(c["sets"], -1, c["rows"], c["hdim"])
    out = y.clone()
    if c["interleaved"]:
        a, b = slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)
    else:
        a, b = slice(0, pairs), slice(c["hdim"] // 2, c["hdim"] // 2 + pairs)
    out[..., a] = y[..., a] * cos - y[..., b] * sin
    out[..., b] = y[..., a] * sin + y[..., b] * cos
    return out.view(x.shape).to(DTYPES[c["dtype"]])


# --------------------------------------------------------------------------------------------- a pass

def run(s):
    c = s["case"]
    if own:
        from paper_2503_15758_amd import binding as a2d
        if c["op"] == "rotary":
            q, k = a2d.rotary((s["Q"], s["K"]), s["positions"], s["freqs"], s["axis"], interleaved=c["interleaved"],
                              inverse=c["inverse"], out_dtype=DTYPES[c["dtype"]])
            return {"Q": q, "K": k}
        rules = {"q_off": c["q_off"], "kv_off": c["kv_off"], "causal": c["causal"], "scale": s["scale"], "softcap": c["cap"],
                 "slopes": s["slopes"], "token_step": c["step"]}
        if c["op"] == "bwd":
            dQ, dK, dV = a2d.partial_bwd_scored(s["Q"], s["K"], s["V"], s["O"], s["dO"], s["lse"], ranges=s["ranges"],
                                                rounded=True, **rules)
            return {"dQ": dQ, "dK": dK, "dV": dV}
        if not c["docs"]:
            O, lse = a2d.partial_fwd_scored(s["Q"], s["K"], s["V"], ranges=s["ranges"], normalised=True, **rules)
            return {"O": O, "lse": lse}
        ranges = a2d.document_ranges(s["starts"], c["nq"], s["prefix"], first=c["q_off"], step=c["step"])
        O, lse = a2d.partial_fwd_scored(s["Q"], s["K"], s["V"], ranges=ranges, normalised=True, **rules)
        return {"O": O, "lse": lse, "ranges": ranges}
    if c["op"] == "rotary":
        return {"Q": _rotated(s, s["Q"]), "K": _rotated(s, s["K"])}
    if c["op"] == "bwd":
        return dict(zip(("dQ", "dK", "dV"), _gradients(s)))
    ranges = _document_ranges(c, s["starts"], s["prefix"]) if c["docs"] else s["ranges"]
    O, lse = _attention(s, ranges)
    return {"O": O, "lse": lse, "ranges": ranges} if c["docs"] else {"O": O, "lse": lse}


# --------------------------------------------------------------------------- what a pass cannot do without

def _seen(c):
    """Keys that each query row sees, row by row (of each sequence)."""
    def keys(first, end):                                       # with tokens in [first, end)
        up = lambda t: min(c["nkv"], max(0, -((c["kv_off"] - t) // c["step"])))
        return max(0, up(end) - up(first))
    far = c["kv_off"] + c["nkv"] * c["step"]
    if c["lens"]:
        return [keys(c["kv_off"], int(n)) for n in c["lens"].split(",") for _ in range(c["nq"])]
    seen = []
    starts, prefix = _documents(c) if c["docs"] else ([], [])
    d = -1
    for i in range(c["nq"]):
        t = c["q_off"] + i * c["step"]
        first, end = c["kv_off"], far
        if c["docs"]:
            while d + 1 < len(starts) and starts[d + 1] <= t:
                d += 1
            first, end = (starts[d], min(starts[d + 1], max(t + 1, starts[d] + prefix[d]))) if 0 <= d < len(prefix) else (0, 0)
        elif c["causal"]:
            end = min(far, t + 1)
        seen.append(keys(first, end))
    return seen


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotary":
        n = (c["heads"] + c["kv_heads"]) * c["rows"] * c["hdim"]
        given = 4 if c["inverse"] else e
        return {"bytes": n * (given + e) + 4 * c["sets"] * c["rows"] * len(c["sections"].split(",")), "flops": 3 * n}
    seen, H = _seen(c), c["hdim"]
    sequences = len(c["lens"].split(",")) if c["lens"] else 1
    scores = sum(seen) * (c["heads"] // sequences)
    # (of a sequence's cache only what it holds has to be read)
    keys = sum(max(seen[b * c["nq"]:(b + 1) * c["nq"]]) for b in range(sequences)) * c["kv_heads"] // sequences if c["lens"] \
        else c["kv_heads"] * c["nkv"]
    q = c["heads"] * c["nq"]
    if c["op"] == "fwd":
        return {"bytes": q * (2 * H * e + 4) + 2 * keys * H * e, "flops": 4 * scores * H}
    # read: Q, O, dO, lse, K, V; written: dQ, dK, dV
    return {"bytes": q * (4 * H * e + 4) + 4 * keys * H * e, "flops": 10 * scores * H}


# ------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rotary":
        p = s["positions"].reshape(c["sets"], -1, c["rows"]).double()
        half = c["hdim"] // 2
        out = {}
        for name in ("Q", "K"):
            y = s[name].double().reshape(c["sets"], -1, c["rows"], c["hdim"]).clone()
            for j in range(s["freqs"].numel()):
                phi = p[:, int(s["axis"][j])].unsqueeze(1) * float(s["freqs"][j]) * (-1.0 if c["inverse"] else 1.0)
                a, b = (2 * j, 2 * j + 1) if c["interleaved"] else (j, half + j)
                z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(phi), phi)
                y[..., a], y[..., b] = z.real, z.imag
            out[name] = y.reshape(s[name].shape)
        return out
    H, group = c["hdim"], c["heads"] // c["kv_heads"]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    t_q = c["q_off"] + torch.arange(c["nq"], **f64) * c["step"]
    t_k = c["kv_off"] + torch.arange(c["nkv"], **f64) * c["step"]
    out, per = {}, c["heads"]
    see = torch.ones(1, c["nq"], c["nkv"], dtype=torch.bool, device="cuda")
    if c["causal"]:
        see &= (t_q.unsqueeze(1) >= t_k.unsqueeze(0))
    if c["docs"]:
        starts, prefix = _documents(c)
        see = torch.zeros_like(see)
        ranges = torch.zeros(c["nq"], 2, dtype=torch.int32, device="cuda")
        for n, first in enumerate(starts[:-1]):
            mine = (t_q >= first) & (t_q < starts[n + 1])
            same = (t_k >= first) & (t_k < starts[n + 1])
            early = t_k < first + prefix[n]
            see |= (mine.unsqueeze(1) & same & (early | (t_k <= t_q.unsqueeze(1)))).unsqueeze(0)
            ranges[mine, 0] = first
            ranges[mine, 1] = (t_q[mine] + 1).clamp(min=first + prefix[n]).clamp(max=starts[n + 1]).int()
        if c["op"] == "fwd":
            out["ranges"] = ranges
    if c["lens"]:
        lens = [int(v) for v in c["lens"].split(",")]
        per = c["heads"] // len(lens)
        see = torch.stack([(t_k < n).unsqueeze(0).expand(c["nq"], -1) for n in lens])
    O = torch.empty(c["heads"], c["nq"], H, **f64)
    lse = torch.empty(c["heads"], c["nq"], **f64)
    dQ, dK, dV = torch.empty_like(O), torch.zeros(c["kv_heads"], c["nkv"], H, **f64), torch.zeros(c["kv_heads"], c["nkv"], H, **f64)
    for h in range(c["heads"]):
        q, k, v = s["Q"][h].double().contiguous(), s["K"][h // group].double().contiguous(), s["V"][h // group].double().contiguous()
        a = torch.mm(q, k.t().contiguous()).mul_(s["scale"])
        if c["cap"]:
            a = a.div_(c["cap"]).tanh_()
            slope_of_cap = 1.0 - a * a if c["op"] == "bwd" else None
            a.mul_(c["cap"])
        if c["slopes"]:
            a -= (t_q.unsqueeze(1) - t_k.unsqueeze(0)).abs_().mul_(float(s["slopes"][h]))
        a.masked_fill_(~see[h // per], -math.inf)
        if c["op"] == "fwd":
            lse[h] = torch.logsumexp(a, 1)
            w = a.sub_(lse[h].unsqueeze(1)).exp_().nan_to_num_(0.0)
            O[h] = torch.mm(w, v)
            continue
        g = s["dO"][h].double().contiguous()
        w = a.sub_(s["lse"][h].double().unsqueeze(1)).exp_().nan_to_num_(0.0)
        ds = w * (torch.mm(g, v.t().contiguous()) - (g * s["O"][h].double()).sum(1, keepdim=True))
        if c["cap"]:
            ds *= slope_of_cap
        ds *= s["scale"]
        dQ[h] = torch.mm(ds, k)
        dK[h // group] += torch.mm(ds.t().contiguous(), q)
        dV[h // group] += torch.mm(w.t().contiguous(), g)
    if c["op"] == "fwd":
        return {"O": O, "lse": lse, **out}
    return {"dQ": dQ, "dK": dK, "dV": dV}
