"""Attention under score rules and rotary positions as they are used: a training step and a serving step of all of them together, sizes
that reach every form of the kernels, calls at the same time, refusals.  Bounds: tests/scored_reference.py."""
import threading

import pytest
import torch

from scored_reference import Scored, half_step, within
from test_gpu_rotary import check, turned
from test_gpu_scored import check_fwd, documents, inputs, int32, slopes_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def a2d():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding
    binding.lib()
    return binding


# ---- sizes that reach the forms of the kernels: workgroups of 256 rows, of 128 in two key lanes, pairs of 128, of 32 in eight key
# lanes with and without parts; dQ in one and two key lanes; key blocks whole, in even parts and shared out; blocks in the order of
# the rows, of the documents' lengths, and more of them than are ranked
LONG = ([0, 500, 501, 700, 1090], [0, 1, 150, 20])
FORMS = [
    ("256 rows", 64, 64, 1024, 260, 128, dict(softcap=20.0)),
    ("256 rows causal", 96, 32, 512, 512, 128, dict(softcap=20.0, causal=True)),
    ("pairs", 64, 64, 1030, 260, 64, dict(slopes=True)),
    ("pairs of documents", 32, 32, 1100, 1090, 64, dict(docs=LONG, slopes=True)),
    ("documents of 256 rows", 16, 16, 1100, 1090, 128, dict(docs=LONG, softcap=9.0)),
    ("two lanes", 14, 7, 1030, 700, 96, dict(softcap=20.0, slopes=True)),
    ("32 rows in parts", 4, 2, 31, 9000, 80, dict(softcap=20.0)),
    ("a token of sequences in parts", 64, 8, 1, 9000, 64, dict(lens=[9000, 4, 8191, 300], slopes=True, q_off=9000)),
    ("causal parts shared out", 8, 4, 1100, 1500, 96, dict(softcap=5.0, causal=True, q_off=400)),
    ("documents shared out", 12, 4, 1100, 1100, 80, dict(docs=([0, 50, 333, 1024, 1090], [0, 0, 400, 0]), slopes=True)),
    ("documents, few rows", 16, 4, 200, 5000, 64, dict(docs=([0, 2400, 2600, 5000], [100, 0, 9]), q_off=2500, softcap=4.0)),
    ("documents, few keys", 5, 5, 9000, 150, 64, dict(docs=([0, 66, 138, 9000], [3, 0, 70]), slopes=True)),
    ("more blocks than are ranked", 1, 1, 135000, 65, 64, dict(docs=([0, 60, 135000], [1, 64]), softcap=20.0)),
    ("more key blocks than are ranked", 1, 1, 70, 135000, 64, dict(docs=([0, 134000, 135000], [9, 0]), q_off=133990)),
    ("one group of many rows", 16, 1, 700, 300, 128, dict(causal=True, slopes=True)),
]


@pytest.mark.parametrize("case", FORMS, ids=lambda c: c[0].replace(" ", "_"))
def test_every_form(a2d, case):
    name, heads, kvh, nq, nkv, H, more = case
    print("scored forms", case, flush=True)
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, "bf16")
    rules = {k: v for k, v in more.items() if k not in ("docs", "lens")}
    if rules.get("slopes"):
        rules["slopes"] = slopes_of(heads)
    if "docs" in more:
        rules["ranges"] = documents(a2d, nq, *more["docs"], first=rules.get("q_off", 0))
    if "lens" in more:
        rules["ranges"] = int32([[[0, n]] * nq for n in more["lens"]])
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    got = a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules)
    check_fwd(got, f, True, Q.dtype, name)
    assert all(torch.equal(x, y) for x, y in zip(got, a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules)))
    if nq == 1:
        return
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    want = s.gradients(O, dO, lse)
    del s, f
    for rounded in (False, True):
        got = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=rounded, **rules)
        for x, n in zip(got, ("dQ", "dK", "dV")):
            within(x, want[n], want["e_" + n], "%s %s" % (name, n), half_step(Q.dtype) if rounded else 0.0)
        again = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=rounded, **rules)
        assert all(torch.equal(x, y) for x, y in zip(got, again)), "not reproducible"
    out = tuple(torch.full_like(x, 1.0, dtype=torch.float32) for x in (Q, K, V))
    plain = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules)
    a2d.partial_bwd_scored(Q, K, V, O, dO, lse, out=out, accumulate=True, **rules)
    # (1 is added first, or last: each of up to 33 partial sums is rounded next to it)
    within(out[0], plain[0].cpu().double() + 1.0, 40 * U * (1.0 + plain[0].cpu().double().abs()), "accumulated")
    assert torch.equal(out[1], plain[1]) and torch.equal(out[2], plain[2])


# ---- a training step: a packed projection, its rotary positions, documents, two tiles of keys and their merge, the gradients
def train(a2d, X, heads, kvh, H, positions, freqs, axis, starts, prefix, rules, dO):
    """X [rows][(heads + 2 kvh) H] -> all that the step leaves"""
    n = X.shape[0]
    qkv = X.view(n, heads + 2 * kvh, H).permute(1, 0, 2)
    q, k, v = qkv[:heads], qkv[heads: heads + kvh], qkv[heads + kvh:]
    q, k = a2d.rotary((q, k), positions, freqs, axis)
    r = a2d.document_ranges(starts, n, prefix)
    cut = n // 2 + 3
    tiles = [(k[:, a:b], v[:, a:b], a) for a, b in ((0, cut), (cut, n))]
    parts = [a2d.partial_fwd_scored(q, kk, vv, kv_off=a, ranges=r, **rules) for kk, vv, a in tiles]
    O, lse = a2d.fix([p[0] for p in parts], [p[1] for p in parts], [p[2] for p in parts], X.dtype)
    dq, dk, dv = None, [], []
    for kk, vv, a in tiles:
        out = (dq if dq is not None else torch.empty(q.shape, device="cuda"), torch.empty(kk.shape, device="cuda"),
               torch.empty(vv.shape, device="cuda"))
        dq, x, y = a2d.partial_bwd_scored(q, kk, vv, O, dO, lse, kv_off=a, ranges=r, out=out, accumulate=dq is not None, **rules)
        dk.append(x)
        dv.append(y)
    dk, dv = torch.cat(dk, 1), torch.cat(dv, 1)
    back = a2d.rotary((dq, dk), positions, freqs, axis, inverse=True, out_dtype=X.dtype)
    return q, k, O, lse, dq, dk, dv, back[0], back[1], r


def steps_inputs(a2d, dt, n, heads, kvh, H, seed=0):
    gen = torch.Generator().manual_seed(seed)
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    X = torch.randn(n, (heads + 2 * kvh) * H, generator=gen).to(dtype).cuda()
    dO = torch.randn(heads, n, H, generator=gen).to(dtype).cuda()
    grid = torch.stack([torch.arange(n) // 49, torch.arange(n) // 7 % 7, torch.arange(n) % 7]).to(torch.int32).cuda()
    freqs, axis = a2d.rotary_frequencies(H, (H // 2 - 2 * (H // 8), H // 8, H // 8))
    return X, dO, grid, freqs, axis, int32([0, 90, 91, n - 20]), int32([40, 0, 100])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_training_step(a2d, dt):
    """Each stage against 64 bits of what it was given; rows of the padding behind the last document have no part in anything.
    In fp32 the whole too: the gradient of the projection against 64-bit automatic differentiation of the formulas."""
    n, heads, kvh, H = 331, 6, 2, 64
    X, dO, pos, freqs, axis, starts, prefix = steps_inputs(a2d, dt, n, heads, kvh, H)
    rules = dict(softcap=6.0, slopes=slopes_of(heads))
    q, k, O, lse, dq, dk, dv, bq, bk, r = train(a2d, X, heads, kvh, H, pos, freqs, axis, starts, prefix, rules, dO)
    qkv = X.view(n, -1, H).permute(1, 0, 2)
    for got, x in ((q, qkv[:heads]), (k, qkv[heads: heads + kvh])):
        check(got, *turned(x, pos, freqs, axis, False, False), X.dtype, "turned")
    s = Scored(q, k, qkv[heads + kvh:], ranges=r, **rules)
    check_fwd((O, lse), {a: b * 2 if a.startswith("e_") else b for a, b in s.partial().items()}, True, X.dtype, "merged")
    want = s.gradients(O, dO, lse)
    for got, name in ((dq, "dQ"), (dk, "dK"), (dv, "dV")):
        within(got, want[name], 2 * want["e_" + name], name)          # (two tiles' roundings)
    for got, x in ((bq, dq), (bk, dk)):
        check(got, *turned(x, pos, freqs, axis, False, True), X.dtype, "turned back")
    assert not bq[:, n - 20:].any() and not bk[:, n - 20:].any() and not dv[:, n - 20:].any() and not O[:, n - 20:].any()
    if dt == "bf16":
        return
    x = X.detach().cpu().double().requires_grad_()
    y = x.view(n, -1, H).permute(1, 0, 2)
    qq, kk = (turned_graph(t, pos, freqs, axis) for t in (y[:heads], y[heads: heads + kvh]))
    kk, vv = kk.repeat_interleave(heads // kvh, 0), y[heads + kvh:].repeat_interleave(heads // kvh, 0)
    z = qq @ kk.transpose(1, 2) / H ** 0.5
    z = 6.0 * torch.tanh(z / 6.0) - slopes_of(heads).cpu().double().view(-1, 1, 1) * (torch.arange(n).view(-1, 1) - torch.arange(n)).abs()
    rr = r.cpu().long()
    see = (torch.arange(n) >= rr[:, :1]) & (torch.arange(n) < rr[:, 1:])
    live = see.any(1)
    p = torch.softmax(z[:, live].masked_fill(~see[live], float("-inf")), 2)
    ((p @ vv) * dO.cpu().double()[:, live]).sum().backward()
    mine = torch.cat([bq, bk, dv]).permute(1, 0, 2).reshape(n, -1).cpu().double()
    # sums of up to n + H terms in fp32 in four products that follow one another (S; P V and dP; dZ; dQ, dK): their worst case, to the whole
    assert (mine - x.grad).norm() <= 4 * (n + H) * U * x.grad.norm()


def turned_graph(x, positions, freqs, axis):
    pos = positions.cpu().double()
    phi = torch.stack([pos[int(axis[p])] * float(freqs[p]) for p in range(freqs.numel())], 1)
    c, s, (a, b) = torch.cos(phi), torch.sin(phi), x.split(x.shape[2] // 2, 2)
    return torch.cat([a * c - b * s, a * s + b * c], 2)


def test_training_step_replayed(a2d):
    """The step captured as a whole: other inputs, documents and positions at every replay, eager work between them."""
    n, heads, kvh, H = 280, 4, 2, 128
    X, dO, pos, freqs, axis, starts, prefix = steps_inputs(a2d, "bf16", n, heads, kvh, H)
    rules = dict(softcap=6.0, slopes=slopes_of(heads))
    step = lambda: train(a2d, X, heads, kvh, H, pos, freqs, axis, starts, prefix, rules, dO)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        X.copy_(steps_inputs(a2d, "bf16", n, heads, kvh, H, seed=i + 1)[0])
        starts.copy_(int32([0, 10 + 60 * i, 200, n - 3 * i]))
        pos.add_(5)
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, eager)), "replay %d" % i


def test_serving_step_replayed(a2d):
    """A token of each of three sequences: its Q and K turned at each sequence's own position, K and V into the cache, attention over
    what each holds by now.  The cache behind the lengths holds NaN; one captured step serves all tokens."""
    seqs, group, kvh, H, room = 3, 4, 2, 128, 500
    heads = group * kvh
    gen = torch.Generator().manual_seed(5)
    rand = lambda *shape: torch.randn(*shape, generator=gen).to(torch.bfloat16).cuda()
    lens = [499, 17, 0]
    K, V = rand(seqs * kvh, room, H), rand(seqs * kvh, room, H)
    for i, n in enumerate(lens):
        K[i * kvh: (i + 1) * kvh, n:] = float("nan")
        V[i * kvh: (i + 1) * kvh, n:] = float("nan")
    x = rand(seqs, heads + 2 * kvh, H)
    at = int32(lens)
    freqs, axis = a2d.rotary_frequencies(H, (64,))
    rows = torch.arange(seqs * kvh, device="cuda")

    def step():
        q = x[:, :heads].reshape(seqs * heads, 1, H)
        k, v = (x[:, a: a + kvh].reshape(seqs * kvh, 1, H) for a in (heads, heads + kvh))
        q, k = a2d.rotary((q, k), at.view(seqs, 1, 1), freqs, axis)
        slot = at.repeat_interleave(kvh).long()
        K.index_put_((rows, slot), k[:, 0])
        V.index_put_((rows, slot), v[:, 0])
        ranges = torch.stack([torch.zeros_like(at), at + 1], 1).view(seqs, 1, 2).contiguous()
        return (q, k) + tuple(a2d.partial_fwd_scored(q, K, V, ranges=ranges, softcap=15.0, normalised=True))

    keep = K.clone(), V.clone()
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    K.copy_(keep[0])
    V.copy_(keep[1])
    for i in range(4):
        if i:
            x.copy_(rand(seqs, heads + 2 * kvh, H))
            at.copy_(int32([499, 17 + i, i]))
        graph.replay()
        torch.cuda.synchronize()
        q, k, O, lse = (t.clone() for t in held)
        check(q, *turned(x[:, :heads].reshape(seqs * heads, 1, H), at.view(seqs, 1, 1), freqs, axis, False, False), torch.bfloat16, "q")
        for n in range(seqs):
            upto = int(at[n]) + 1
            kk, vv = (t[n * kvh: (n + 1) * kvh, :upto] for t in (K, V))
            ref = Scored(q[n * heads: (n + 1) * heads], kk, vv, softcap=15.0).partial()
            check_fwd((O[n * heads: (n + 1) * heads], lse[n * heads: (n + 1) * heads]), ref, True, torch.bfloat16, "sequence %d" % n)


def test_two_streams_and_threads_at_once(a2d):
    """Calls with partials of their own, from two threads on two streams: each gets what it gets alone."""
    jobs = []
    for seed, (heads, kvh, nq, nkv, H) in enumerate([(8, 1, 300, 2100, 128), (4, 2, 1, 6000, 64)]):
        Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, "bf16", seed=seed)
        rules = dict(softcap=8.0, slopes=slopes_of(heads), causal=True, q_off=nkv - nq)

        def job(Q=Q, K=K, V=V, dO=dO, rules=rules):
            O, lse = a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules)
            return (O, lse) + tuple(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=True, **rules))
        jobs.append(job)
    want = [j() for j in jobs]
    torch.cuda.synchronize()
    got, streams = [None, None], [torch.cuda.Stream(), torch.cuda.Stream()]

    def run(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(10):
                got[i] = jobs[i]()
    threads = [threading.Thread(target=run, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(x, y) for x, y in zip(want[i], got[i])), i


def test_the_same_tensor_twice(a2d):
    """Queries that are the keys, and values that are the keys too."""
    X = inputs(2, 2, 150, 150, 64, "bf16")[0]
    rules = dict(softcap=3.0, causal=True)
    check_fwd(a2d.partial_fwd_scored(X, X, X, normalised=True, **rules), Scored(X, X, X, **rules).partial(), True, X.dtype, "one tensor")
    with pytest.raises(a2d.A2DError):
        a2d.rotary((X, X), int32([list(range(150))]), *a2d.rotary_frequencies(64, (32,)), out=(X, X))


def test_refusals(a2d):
    refused = (a2d.A2DError, ValueError)             # (of another number of tensors: ValueError)
    heads, kvh, nq, nkv, H = 4, 2, 20, 30, 64
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, "bf16")
    O, lse = a2d.partial_fwd_scored(Q, K, V, normalised=True)
    f32 = lambda *shape: torch.zeros(*shape, device="cuda")
    ok = dict(ranges=int32([[0, 30]] * nq), slopes=slopes_of(heads))
    bad = [dict(slopes=f32(heads).double()), dict(slopes=f32(kvh)), dict(slopes=f32(2 * heads)[::2]), dict(slopes=f32(heads).cpu()),
           dict(ranges=ok["ranges"][:-1]), dict(ranges=ok["ranges"].long()), dict(ranges=ok["ranges"].cpu()),
           dict(ranges=ok["ranges"].expand(3, nq, 2).contiguous()), dict(ranges=ok["ranges"].expand(2, nq, 2)),
           dict(softcap=-1.0), dict(softcap=float("nan")), dict(token_step=0), dict(token_step=1 << 40), dict(scale=-1.0),
           dict(q_off=1 << 30, slopes=ok["slopes"])]
    for change in bad:
        with pytest.raises(refused):
            a2d.partial_fwd_scored(Q, K, V, **{**ok, **change})
        with pytest.raises(refused):
            a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **{**ok, **change})
    row = Q[:1, :1]
    wrong = [(Q, K, V[:, :-1]), (Q, K.float(), V.float()), (Q[:3], K, V), (Q, K, V.cpu()), (Q[:, :, :48], K[:, :, :48], V[:, :, :48]),
             (row.expand(heads, nq, H), K, V), (Q, K[:1, :1].expand(kvh, nkv, H), V), (Q, K[:, :1].expand(kvh, nkv, H), V),
             (Q.half(), K.half(), V.half())]
    for q, k, v in wrong:
        with pytest.raises(refused):
            a2d.partial_fwd_scored(q, k, v)
    for out in ((f32(heads, nq, H), f32(heads, nq)), (f32(heads, nq, H), f32(heads, nq), f32(heads, nq - 1)),
                (f32(heads, nq, H), f32(heads, nq), f32(nq, heads).t())):
        with pytest.raises(refused):
            a2d.partial_fwd_scored(Q, K, V, out=out)
    with pytest.raises(refused):
        a2d.partial_fwd_scored(Q, K, V, accumulate=True)
    with pytest.raises(refused):
        a2d.partial_fwd_scored(Q, K, V, out=(O, lse), accumulate=True, normalised=True)
    for o, g, l in ((O.float(), dO, lse), (O, dO[:, :-1], lse), (O, dO, lse.t().contiguous().t()), (O, dO, lse[:, :-1])):
        with pytest.raises(refused):
            a2d.partial_bwd_scored(Q, K, V, o, g, l)
    with pytest.raises(refused):
        a2d.partial_bwd_scored(Q, K, V, O, dO, lse, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(refused):
        a2d.partial_bwd_scored(Q, K, V, O, dO, lse, out=(f32(heads, nq, H),) * 2 + (f32(heads, nkv, H),))
    freqs, axis = a2d.rotary_frequencies(H, (32,))
    pos = int32([list(range(nq))])
    for args, kw in (((row.expand(heads, nq, H), pos, freqs), {}), ((Q, pos[:, 1:], freqs), {}), ((Q, pos.long(), freqs), {}),
                     ((Q, pos, freqs.float()), {}), ((Q, pos, freqs.cuda()), {}), ((Q, pos, freqs, axis + 1), {}), ((Q, pos, freqs, axis[1:]), {}),
                     ((Q, pos, freqs, axis), dict(out=Q[:, :, :32])), ((Q, pos, freqs, axis), dict(out=Q.float())),
                     (((Q, Q[:, 1:]), pos, freqs), {}), (((Q, K[:, :nq].float()), pos, freqs), {}), (((Q, Q, Q), pos, freqs), {}),
                     ((Q, pos.expand(3, 1, nq).contiguous(), freqs), {}), ((Q.cpu(), pos, freqs), {}), ((Q, pos, freqs), dict(out_dtype=torch.float32))):
        with pytest.raises(refused):
            a2d.rotary(*args, **kw)
    for args, kw in (((int32([0]), 5), {}), ((int32([[0, 5]]), 5), {}), ((int32([0, 5]).long(), 5), {}), ((int32([0, 5]), 0), {}),
                     ((int32([0, 5]), 5, int32([1, 1])), {}), ((int32([0, 5]), 5), dict(step=0)), ((int32([0, 5]), 5), dict(out=int32([[0, 0]]))),
                     ((int32([0, 5]).cpu(), 5), {})):
        with pytest.raises(refused):
            a2d.document_ranges(*args, **kw)
    torch.cuda.synchronize()


def test_frequencies_of_any_size(a2d):
    """Parts of a turn from frequencies of either sign, from ones that never get anywhere to some turns a position, against angles from
    rational arithmetic: position times frequency is exact there, and 2 pi is good to 300 bits."""
    import math
    from fractions import Fraction

    def arctan(x):                                   # of 1 / x, in units of 2^-300
        total = term = (1 << 300) // x
        n, sign = 3, -1
        while term:
            term //= x * x
            total += sign * (term // n)
            n, sign = n + 2, -sign
        return total

    turn = Fraction(8 * (4 * arctan(5) - arctan(239)), 1 << 300)
    f = [1.0, -1.0, 0.1, -1e-4, 1e-30, -5e-324, 6.283185307179586, 1e3, -123456.789, 1e9, 0.0, 2.0 ** -33]
    rows = [0, 1, -1, 77, 2 ** 31 - 1, -2 ** 31]
    X = torch.zeros(1, len(rows), 32, device="cuda")
    X[:, :, :16] = 1.0
    got = a2d.rotary(X, int32([rows]), torch.tensor(f, dtype=torch.float64)).cpu().double()
    for i, n in enumerate(rows):
        for p, freq in enumerate(f):
            part = float((n * Fraction(freq) / turn) % 1)
            want = (math.cos(2 * math.pi * part), math.sin(2 * math.pi * part))
            # 2^-64 turns a position, the angle's 2^-32 turns and its fp32 rounding (half a turn at most), 4 half steps of the sine
            bound = 2 * math.pi * (abs(n) * 2.0 ** -64 + 2.0 ** -32 + 2.0 ** -25) + 4 * U
            assert abs(got[0, i, p] - want[0]) <= bound and abs(got[0, i, 16 + p] - want[1]) <= bound, (n, freq)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("step, slopes", [(1, [8.0, 0.5, -0.01, 1e-6]), (1000, [0.01, 1e-4, 3.0, 0.0]), (4, [30.0, -0.25, 0.0, 0.125])])
def test_steep_and_rising_slopes(a2d, dt, step, slopes):
    """Rows with keys on both sides, and a bias that changes within a block by more than fp32 could forget, or rises with distance."""
    Q, K, V, dO = inputs(4, 2, 330, 470, 64, dt)
    rules = dict(slopes=torch.tensor(slopes, device="cuda"), token_step=step, q_off=70 * step + step // 2)
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    check_fwd(a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules), f, True, Q.dtype, "slopes")
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    want = s.gradients(O, dO, lse)
    for x, n in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules), ("dQ", "dK", "dV")):
        within(x, want[n], want["e_" + n], "slopes %s" % n)


@pytest.mark.parametrize("dt, kvh, nq", [("bf16", 5, 1), ("bf16", 2, 40), ("f32", 2, 3)])
def test_a_long_cache(a2d, dt, kvh, nq):
    """4 million keys a head, so that heads begin beyond 4 GiB: sequences that see runs at its start, across its middle and at its end, and
    the rest of it as it was allocated; the gradients of what no row sees are zeros."""
    nkv, H, group = (1 << 22) - 3, 128, 2
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(2)
    rand = lambda *shape: torch.randn(*shape, generator=gen).to(dtype).cuda()
    K, V = (torch.empty(kvh, nkv, H, dtype=dtype, device="cuda") for _ in range(2))
    Q, dO = rand(kvh * group, nq, H), rand(kvh * group, nq, H)
    seen = [((i * (nkv - 300)) // max(kvh - 1, 1), (i * (nkv - 300)) // max(kvh - 1, 1) + 300) for i in range(kvh)]
    for i, (a, b) in enumerate(seen):
        K[i, a:b], V[i, a:b] = rand(b - a, H), rand(b - a, H)
    rules = dict(softcap=9.0)
    ranges = int32([[list(x)] * nq for x in seen])
    O, lse = a2d.partial_fwd_scored(Q, K, V, ranges=ranges, normalised=True, **rules)
    refs = [Scored(Q[i * group: (i + 1) * group], K[i: i + 1, a:b], V[i: i + 1, a:b], **rules) for i, (a, b) in enumerate(seen)]
    for i, s in enumerate(refs):
        h = slice(i * group, (i + 1) * group)
        check_fwd((O[h], lse[h]), s.partial(), True, dtype, "sequence %d" % i)
    if kvh > 2:
        return
    dQ, dK, dV = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, ranges=ranges, rounded=True, **rules)
    for i, (a, b) in enumerate(seen):
        h = slice(i * group, (i + 1) * group)
        want = refs[i].gradients(O[h], dO[h], lse[h])
        for got, n in ((dQ[h], "dQ"), (dK[i: i + 1, a:b], "dK"), (dV[i: i + 1, a:b], "dV")):
            within(got, want[n], want["e_" + n], n, half_step(dtype) or U)
        for x in (dK, dV):
            assert not x[i, :a].any() and not x[i, b:].any()
    with pytest.raises(a2d.A2DError):                # rows of a head that span 4 GiB
        a2d.partial_fwd_scored(Q, torch.empty(nkv, 5, H, dtype=dtype, device="cuda").permute(1, 0, 2)[:kvh],
                               torch.empty(nkv, 5, H, dtype=dtype, device="cuda").permute(1, 0, 2)[:kvh])


@pytest.mark.parametrize("case", [c for c in FORMS if c[3] < 10000 and c[4] > 1], ids=lambda c: c[0].replace(" ", "_"))
def test_every_form_accumulated(a2d, case):
    """Two tiles of keys, views of one cache, the second continuing the first's partial: the whole's, at every form."""
    name, heads, kvh, nq, nkv, H, more = case
    print("scored forms accumulated", case, flush=True)
    Q, K, V, _ = inputs(heads, kvh, nq, nkv, H, "bf16")
    rules = {k: v for k, v in more.items() if k not in ("docs", "lens")}
    if rules.get("slopes"):
        rules["slopes"] = slopes_of(heads)
    if "docs" in more:
        rules["ranges"] = documents(a2d, nq, *more["docs"], first=rules.get("q_off", 0))
    if "lens" in more:
        rules["ranges"] = int32([[[0, n]] * nq for n in more["lens"]])
    cut = nkv // 3 + 5
    out = a2d.partial_fwd_scored(Q, K[:, cut:], V[:, cut:], kv_off=cut, **rules)
    a2d.partial_fwd_scored(Q, K[:, :cut], V[:, :cut], out=out, accumulate=True, **rules)
    ref = Scored(Q, K, V, **rules).partial()
    check_fwd(out, {k: v * 2 if k.startswith("e_") else v for k, v in ref.items()}, False, Q.dtype, name)


@pytest.mark.parametrize("dt, nq, kvh", [("bf16", 200, 2), ("f32", 200, 2), ("bf16", 7, 1), ("bf16", 300, 4)])
@pytest.mark.parametrize("step, q_off, kv_off", [(1, 0, 0), (3, 1, 2), (1, -40, -20), (7, 1 << 20, (1 << 20) - 300)])
def test_ranges_of_any_kind(a2d, dt, nq, kvh, step, q_off, kv_off):
    """Ranges that end before they begin, hold nothing, lie in front of or behind all keys, or span every token there is."""
    heads, nkv = 4, 333
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, 64, dt)
    end = kv_off + nkv * step
    kinds = [(-2 ** 31, 2 ** 31 - 1), (kv_off + 10, kv_off + 5), (-50, kv_off + 20), (end + 5, end + 90), (kv_off + 11, kv_off + 12), (0, 0),
             (kv_off - 9, kv_off), (end - step, 2 ** 31 - 1), (2 ** 31 - 1, -2 ** 31), (kv_off + 30, end - 40), (-1, 2 ** 31 - 1)]
    gen = torch.Generator().manual_seed(nq)
    sets = torch.tensor(kinds, dtype=torch.int32)[torch.randint(0, len(kinds), (kvh, nq), generator=gen)].cuda()
    for ranges, causal in ((sets, False), (sets[0].contiguous(), True)):
        rules = dict(ranges=ranges, causal=causal, q_off=q_off, kv_off=kv_off, token_step=step, softcap=12.0, slopes=slopes_of(heads) / step)
        s = Scored(Q, K, V, **rules)
        f = s.partial()
        check_fwd(a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules), f, True, Q.dtype, "ranges")
        O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
        want = s.gradients(O, dO, lse)
        for x, n in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules), ("dQ", "dK", "dV")):
            within(x, want[n], want["e_" + n], "ranges %s" % n)


@pytest.mark.parametrize("dt, heads, kvh, nq", [("bf16", 65535, 65535, 1), ("bf16", 65535, 13107, 2), ("f32", 65535, 21845, 2), ("bf16", 65520, 65520, 40)])
def test_as_many_heads_as_there_may_be(a2d, dt, heads, kvh, nq):
    Q, K, V, dO = inputs(heads, kvh, nq, 3, 64, dt)
    rules = dict(softcap=5.0, slopes=torch.rand(heads, generator=torch.Generator().manual_seed(1)).cuda(), causal=True, q_off=1)
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    check_fwd(a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules), f, True, Q.dtype, "heads")
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    want = s.gradients(O, dO, lse)
    for x, n in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=True, **rules), ("dQ", "dK", "dV")):
        within(x, want[n], want["e_" + n], "heads %s" % n, half_step(Q.dtype) or U)
    freqs, axis = a2d.rotary_frequencies(64, (16, 16))
    pos = torch.arange(2 * nq, dtype=torch.int32, device="cuda").view(2, nq)
    check(a2d.rotary(Q, pos, freqs, axis), *turned(Q, pos, freqs, axis, False, False), Q.dtype, "turned")
