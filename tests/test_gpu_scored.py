"""Attention under score rules (a tanh cap, a distance bias, ranges of tokens) against 64 bits: forward, backward, the call
forms, what masked places hold.  Bounds: tests/scored_reference.py, by element."""
import itertools
import math

import pytest
import torch

from scored_reference import Scored, half_step, within

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", params=["default", "generic"])
def a2d(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding
    binding.lib()
    binding.force_generic(request.param == "generic")
    yield binding
    binding.force_generic(False)


def rand(gen, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float32) * sigma).to(dtype).cuda()


def heads_of(gen, heads, rows, H, dtype, packed=False, sigma=1.0):
    if packed:
        return rand(gen, (rows, heads, H), dtype, sigma).permute(1, 0, 2)
    return rand(gen, (heads, rows, H), dtype, sigma)


def inputs(heads, kvh, nq, nkv, H, dt, packed=False, sigma=1.0, seed=0):
    gen = torch.Generator().manual_seed(1000 + seed)
    dtype = DT[dt]
    return (heads_of(gen, heads, nq, H, dtype, packed, sigma), heads_of(gen, kvh, nkv, H, dtype, packed),
            heads_of(gen, kvh, nkv, H, dtype, packed), heads_of(gen, heads, nq, H, dtype, packed))


def slopes_of(heads):
    return torch.exp2(-8.0 * torch.arange(1, heads + 1, dtype=torch.float32) / heads).cuda()


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def documents(a2d, nq, starts, prefix, **more):
    return a2d.document_ranges(int32(starts), nq, int32(prefix) if prefix else None, **more)


# heads, kv_heads, nq, nkv, H, type, rules; "docs": (starts, prefix)
DOCS = ([0, 70, 70, 133, 290], [10, 0, 63, 150])
CASES = [
    ("cap", 2, 2, 128, 128, 128, "bf16", dict(softcap=20.0)),
    ("cap causal", 4, 2, 200, 300, 64, "bf16", dict(softcap=5.0, causal=True, q_off=100)),
    ("bias", 4, 4, 257, 129, 96, "bf16", dict(slopes=True)),
    ("bias causal", 8, 2, 130, 190, 80, "bf16", dict(slopes=True, causal=True, q_off=60)),
    ("cap bias", 4, 1, 65, 513, 128, "bf16", dict(softcap=8.0, slopes=True, q_off=1000, kv_off=900)),
    ("cap bias causal", 3, 3, 300, 300, 128, "bf16", dict(softcap=8.0, slopes=True, causal=True)),
    ("documents", 2, 2, 300, 300, 64, "bf16", dict(docs=DOCS)),
    ("documents cap bias", 6, 2, 300, 300, 128, "bf16", dict(docs=DOCS, softcap=15.0, slopes=True)),
    ("documents of a tile", 2, 1, 100, 150, 96, "bf16", dict(docs=DOCS, q_off=120, kv_off=60, slopes=True)),
    ("cyclic", 2, 2, 150, 150, 128, "bf16", dict(causal=True, q_off=2, kv_off=3, token_step=4, slopes=True)),
    ("cyclic documents", 2, 2, 100, 90, 80, "bf16", dict(docs=([0, 100, 301, 400], [50, 0, 20]), q_off=1, kv_off=2, token_step=4)),
    ("one token", 8, 2, 1, 1, 128, "bf16", dict(softcap=10.0, slopes=True)),
    ("one row", 16, 2, 1, 1000, 128, "bf16", dict(softcap=10.0, lens=[1000])),
    ("one row of sequences", 24, 6, 1, 700, 64, "bf16", dict(lens=[700, 1, 333], slopes=True, q_off=700)),
    ("three rows of sequences", 12, 4, 3, 260, 96, "bf16", dict(lens=[100, 0], softcap=30.0)),
    ("one key", 2, 2, 100, 1, 128, "bf16", dict(slopes=True)),
    ("large tile", 2, 1, 520, 1500, 128, "bf16", dict(softcap=30.0, causal=True, q_off=980, sigma=3.0)),
    ("saturated cap", 2, 2, 140, 200, 64, "bf16", dict(softcap=2.0, sigma=20.0)),
    ("wide cap", 2, 2, 140, 200, 128, "bf16", dict(softcap=1e6)),
    ("packed", 6, 2, 131, 67, 80, "bf16", dict(softcap=20.0, slopes=True, causal=True, packed=True)),
    ("nothing seen", 2, 2, 64, 64, 128, "bf16", dict(causal=True, kv_off=64, softcap=5.0)),
    ("far", 2, 2, 64, 64, 128, "bf16", dict(causal=True, q_off=(1 << 35) + 20, kv_off=1 << 35, slopes=True)),
    ("fp32 cap", 2, 2, 128, 128, 64, "f32", dict(softcap=20.0)),
    ("fp32 all", 6, 2, 150, 203, 96, "f32", dict(softcap=7.0, slopes=True, causal=True, q_off=53)),
    ("fp32 documents", 2, 2, 300, 300, 128, "f32", dict(docs=DOCS, slopes=True)),
    ("fp32 one row", 8, 2, 1, 400, 80, "f32", dict(lens=[399], softcap=20.0)),
    ("fp32 wide cap", 2, 2, 70, 100, 64, "f32", dict(softcap=1e6)),
    ("fp32 cyclic packed", 4, 4, 77, 99, 128, "f32", dict(docs=([0, 100, 390], [30, 0]), q_off=3, kv_off=0, token_step=4, packed=True)),
]


def problem(a2d, case, seed=0):
    name, heads, kvh, nq, nkv, H, dt, more = case
    rules = {k: v for k, v in more.items() if k not in ("docs", "lens", "packed", "sigma")}
    t = inputs(heads, kvh, nq, nkv, H, dt, more.get("packed", False), more.get("sigma", 1.0), seed)
    if rules.get("slopes"):
        rules["slopes"] = slopes_of(heads)
    if "docs" in more:
        rules["ranges"] = documents(a2d, nq, *more["docs"], first=rules.get("q_off", 0), step=rules.get("token_step", 1))
    if "lens" in more:
        rules["ranges"] = int32([[[0, n]] * nq for n in more["lens"]])
    return t, rules


def check_fwd(got, ref, norm, dtype, what):
    r = half_step(dtype)
    if norm:
        O, lse = got
        within(O, ref["O"], ref["e_O"], what + " O", r)
    else:
        N, m, l = (x.detach().cpu().double() for x in got)
        assert not torch.isnan(N).any() and not torch.isnan(m).any() and not torch.isnan(l).any(), what
        some = l > 0
        assert torch.equal(some, ref["l"] > 0), what + ": empty rows"
        assert torch.equal(m[~some], torch.full_like(m[~some], -math.inf)) and not N[~some].any() and not l[~some].any(), what
        within(m, ref["m"], ref["e_m"], what + " m")
        within(torch.where(some.unsqueeze(2), N / torch.where(some, l, torch.ones_like(l)).unsqueeze(2), torch.zeros_like(N)),
               ref["O"], ref["e_O"], what + " N / l")
        lse = torch.where(some, m + torch.log(torch.where(some, l, torch.ones_like(l))), torch.full_like(l, -math.inf))
    within(lse, ref["lse"], ref["e_lse"], what + " lse")


@pytest.mark.parametrize("case", CASES, ids=lambda c: c[0].replace(" ", "_"))
def test_forward(a2d, case):
    (Q, K, V, _), rules = problem(a2d, case)
    print("scored forward", case, flush=True)
    ref = Scored(Q, K, V, **rules).partial()
    for norm in (False, True):
        got = a2d.partial_fwd_scored(Q, K, V, normalised=norm, **rules)
        check_fwd(got, ref, norm, Q.dtype, case[0])
        again = a2d.partial_fwd_scored(Q, K, V, normalised=norm, **rules)
        assert all(torch.equal(x, y) for x, y in zip(got, again)), "not reproducible"


@pytest.mark.parametrize("case", CASES, ids=lambda c: c[0].replace(" ", "_"))
def test_backward(a2d, case):
    (Q, K, V, dO), rules = problem(a2d, case)
    print("scored backward", case, flush=True)
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    if not dO.is_contiguous():
        O = torch.empty_like(dO).copy_(O)
    ref = s.gradients(O, dO, lse)
    for rounded in (False, True):
        got = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=rounded, **rules)
        for x, name in zip(got, ("dQ", "dK", "dV")):
            within(x, ref[name], ref["e_" + name], "%s %s" % (case[0], name), half_step(Q.dtype) if rounded else 0.0)
        again = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=rounded, **rules)
        assert all(torch.equal(x, y) for x, y in zip(got, again)), "not reproducible"


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_accumulated_over_key_blocks(a2d, dt):
    """Three key blocks, the middle one of another document: partials added up in place, their merge, and the gradients'
    sums are those of the whole."""
    heads, kvh, nq, H = 4, 2, 150, 128
    Q, K, V, dO = inputs(heads, kvh, nq, 330, H, dt)
    rules = dict(softcap=9.0, slopes=slopes_of(heads), scale=0.1)
    ranges = documents(a2d, nq, [0, 100, 200, 330], [0, 40, 300], first=180)
    s = Scored(Q, K, V, q_off=180, ranges=ranges, **rules)
    ref = s.partial()
    cuts, parts, acc = [0, 90, 210, 330], [], None
    for a, b in zip(cuts, cuts[1:]):
        k, v = K[:, a:b].contiguous(), V[:, a:b].contiguous()
        parts.append(a2d.partial_fwd_scored(Q, k, v, q_off=180, kv_off=a, ranges=ranges, **rules))
        if acc is None:
            acc = tuple(x.clone() for x in parts[0])
        else:
            a2d.partial_fwd_scored(Q, k, v, q_off=180, kv_off=a, ranges=ranges, out=acc, accumulate=True, **rules)
    check_fwd(acc, {k: v * 2 if k.startswith("e_") else v for k, v in ref.items()}, False, Q.dtype, "accumulated")
    O, lse = a2d.fix([p[0] for p in parts], [p[1] for p in parts], [p[2] for p in parts], Q.dtype)
    check_fwd((O, lse), {k: v * 2 if k.startswith("e_") else v for k, v in ref.items()}, True, Q.dtype, "merged")
    want = s.gradients(O, dO, lse)
    dQ = torch.full((heads, nq, H), 1.0, device="cuda")
    dk, dv = [], []
    for a, b in zip(cuts, cuts[1:]):
        k, v = K[:, a:b].contiguous(), V[:, a:b].contiguous()
        out = (dQ, torch.empty_like(k, dtype=torch.float32), torch.empty_like(v, dtype=torch.float32))
        a2d.partial_bwd_scored(Q, k, v, O, dO, lse, q_off=180, kv_off=a, ranges=ranges, out=out, accumulate=True, **rules)
        dk.append(out[1])
        dv.append(out[2])
    within(dQ, want["dQ"] + 1.0, want["e_dQ"] + 8 * 2.0 ** -24 * (1 + want["dQ"].abs()), "dQ")
    within(torch.cat(dk, 1), want["dK"], want["e_dK"], "dK")
    within(torch.cat(dv, 1), want["dV"], want["e_dV"], "dV")


@pytest.mark.parametrize("dt, nq", [("bf16", 300), ("f32", 300), ("bf16", 5)])
def test_what_nobody_sees_may_hold_anything(a2d, dt, nq):
    """Padding rows, and keys in front of and behind all that is seen: NaN and infinities there change nothing, and their
    gradients are 0."""
    heads, kvh, nkv, H = 4, 2, 500, 128
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, dt)
    # rows from `pad` on see nothing; keys 37 .. 411 are seen
    pad = nq - nq // 4
    t = torch.zeros(nq, 2, dtype=torch.int32)
    t[:, 0], t[:, 1] = 37, 412
    t[: nq // 2, 1] = 200
    t[pad:] = 0
    rules = dict(softcap=12.0, slopes=slopes_of(heads), ranges=t.cuda())
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    want = s.gradients(O, dO, lse)
    for fill in (float("nan"), float("inf"), float("-inf")):
        q, k, v, g, o = (x.clone() for x in (Q, K, V, dO, O))
        for x in (q, g, o):
            x[:, pad:] = fill
        for x in (k, v):
            x[:, :37] = fill
            x[:, 412:] = fill
        check_fwd(a2d.partial_fwd_scored(q, k, v, normalised=True, **rules), f, True, Q.dtype, "filled")
        got = a2d.partial_bwd_scored(q, k, v, o, g, lse, **rules)
        for x, name in zip(got, ("dQ", "dK", "dV")):
            within(x, want[name], want["e_" + name], "%s (%s)" % (name, fill))
        assert not got[0][:, pad:].any() and not got[1][:, :37].any() and not got[2][:, 412:].any()


def test_a_hidden_score_may_overflow(a2d):
    """Scores of infinite size behind the mask, or NaN ones of a key that only later rows see: nothing of them comes through."""
    Q, K, V, dO = inputs(2, 2, 128, 128, 64, "bf16")
    K[:, 100:] = 3e38
    rules = dict(softcap=10.0, causal=True)
    s = Scored(Q[:, :100], K[:, :100], V[:, :100], **rules)
    f = s.partial()
    O, lse = a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules)
    check_fwd((O[:, :100], lse[:, :100]), f, True, Q.dtype, "overflow")


def test_gradient_against_differences(a2d):
    """d loss / d x of Q, K and V in fp32 against central differences of the forward's own outputs in 64 bits."""
    heads, kvh, nq, nkv, H = 2, 1, 20, 33, 64
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, "f32")
    rules = dict(softcap=3.0, slopes=slopes_of(heads), ranges=documents(a2d, nq, [0, 7, 40], [5, 3]))
    O, lse = a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules)
    got = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules)
    g64, step = dO.cpu().double(), 1e-5
    gen = torch.Generator().manual_seed(3)
    for which, grad in enumerate(got):
        for _ in range(4):
            d = torch.randn(grad.shape, generator=gen, dtype=torch.float64)
            loss = []
            for sign in (1, -1):
                x = [t.cpu().double() for t in (Q, K, V)]
                x[which] = x[which] + sign * step * d
                loss.append((Scored(*x, **rules).partial()["O"] * g64).sum().item())
            # (the difference's own error: step^2 of a third derivative, and 2^-52 of the sums over the step)
            want, mine = (loss[0] - loss[1]) / (2 * step), (grad.cpu().double() * d).sum().item()
            assert abs(mine - want) <= 1e-4 * (grad.cpu().double().abs() * d.abs()).sum().item(), (which, mine, want)


@pytest.mark.parametrize("first, step, rows, causal", [(0, 1, 300, True), (-5, 1, 320, True), (3, 7, 60, True), (0, 1, 300, False),
                                                       ((1 << 31) - 20, 3, 30, True), (250, 1, 1, True)])
def test_document_ranges(a2d, first, step, rows, causal):
    starts, prefix = [0, 5, 5, 100, 130, 290], [2, 9, 0, 500, -3]
    got = a2d.document_ranges(int32(starts), rows, int32(prefix), first=first, step=step, causal=causal).cpu().tolist()
    for i, pair in enumerate(got):
        t, want = first + i * step, [0, 0]
        for d in range(5):
            if starts[d] <= t < starts[d + 1]:
                want = [starts[d], min(starts[d + 1], max(t + 1, starts[d] + prefix[d])) if causal else starts[d + 1]]
        assert pair == want, (i, t)


def test_on_another_stream_and_replayed(a2d):
    """The calls go to the current stream, and a captured run of them gives the eager results at every replay."""
    heads, kvh, n, H = 4, 2, 270, 128
    Q, K, V, dO = inputs(heads, kvh, n, n, H, "bf16")
    rules = dict(softcap=20.0, slopes=slopes_of(heads))
    starts, prefix = int32([0, 100, 250]), int32([30, 0])

    def both():
        r = a2d.document_ranges(starts, n, prefix)
        O, lse = a2d.partial_fwd_scored(Q, K, V, ranges=r, normalised=True, **rules)
        return (O, lse) + tuple(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, ranges=r, **rules))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        here = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(want, here))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        Q.copy_(inputs(heads, kvh, n, n, H, "bf16", seed=i + 1)[0])
        eager = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, eager)), "replay %d" % i
