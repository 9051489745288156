"""The paged cache and the attention over it as programs use them: steps of serving, shares of a text, streams, graphs, views,
caches of more than 4 GiB, and what may hold anything."""
import ctypes
import math

import pytest
import torch

import cached_reference as ref
from paper_2503_15758_amd import binding as a2d
from test_gpu_cached_attention import _call, _check, _expect, _problem

pytestmark = pytest.mark.gpu

FORMATS = {"bf16": a2d.CACHE_BF16, "e4m3": a2d.CACHE_E4M3, "e2m1": a2d.CACHE_E2M1}


def _same(x, y):
    return all(torch.equal(a, b) for a, b in zip(x, y))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "e2m1"])
def test_serving(fmt):
    """Prompts are written; a few times a tree is drafted, placed, turned, seen, and one of its paths kept; and all is read back for the
    tile calls, which see the same."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, heads, kv_heads, H, page_rows, columns, rows = 3, 8, 2, 128, 32, 8, 9
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    cache = a2d.cache_empty(n * columns, kv_heads, page_rows, H, FORMATS[fmt])
    for x in cache[:2]:                                     # (nothing is cleared: unwritten tokens are NaN or anything)
        (x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)).fill_(-1 if x.element_size() == 2 else 255)
    table = torch.randperm(n * columns, generator=gen, device="cuda").view(n, columns).int()
    lens = torch.tensor([100, 1, 57], dtype=torch.int32, device="cuda")
    prompt = [normal(n, 100, kv_heads, H).permute(0, 2, 1, 3) for _ in range(2)]
    tokens = torch.arange(100, device="cuda", dtype=torch.int32)
    index = torch.where(tokens < lens.unsqueeze(1), tokens, -1)
    a2d.cache_write(cache, table, *prompt, torch.zeros_like(lens), index=index)
    freqs, axis = a2d.rotary_frequencies(H, [H // 2])
    for step in range(3):
        parents = torch.tensor([[-1, 0, 0, 1, 1, 2, 5, 6, 7]] * 2 + [[-1, 0, 1, 2, -2, -2, -2, -2, -2]], dtype=torch.int32, device="cuda")
        masks, positions = a2d.tree_masks(parents, lens)
        Q, K, V = normal(n, heads, rows, H), normal(n, kv_heads, rows, H), normal(n, kv_heads, rows, H)
        Q, K = (x.view_as(y) for x, y in zip(a2d.rotary((Q.view(-1, rows, H), K.view(-1, rows, H)), positions, freqs, axis), (Q, K)))
        O, lse = a2d.partial_fwd_cached(Q, cache, table, lens, K, V, masks, max_tokens=n * columns, normalised=True)
        x = {"cache": cache, "table": table.cpu(), "lens": lens.cpu(), "Q": Q, "K": K, "V": V, "masks": masks.cpu(), "scale": 1 / math.sqrt(H)}
        _check(x)
        assert bool(torch.isfinite(O).all())
        # the longest path is kept: rows 0, 2, 5, 6 of two sequences, 0, 1 of the last
        keep = torch.tensor([[0, 2, 5, 6]] * 2 + [[0, 1, -1, -1]], dtype=torch.int32, device="cuda")
        a2d.cache_write(cache, table, K, V, lens, index=keep)
        lens = lens + (keep >= 0).sum(1).int()
    K, V = a2d.cache_read(cache, table, lens, 112)
    assert bool(torch.isfinite(K).all()) and bool(torch.isfinite(V).all())
    Q = normal(n, heads, 1, H)
    O, lse = a2d.partial_fwd_cached(Q, cache, table, lens, normalised=True)
    ranges = torch.stack([torch.zeros_like(lens), lens], 1).view(n, 1, 2).contiguous()
    O2, lse2 = a2d.partial_fwd_scored(Q.view(-1, 1, H), K.reshape(-1, 112, H), V.reshape(-1, 112, H), ranges=ranges, normalised=True)
    # (both are within their bounds of the same numbers)
    values = [ref.cache_values(cache, i) for i in range(2)]
    got = ref.attention(Q, values, table.cpu(), lens.cpu(), scale=1 / math.sqrt(H))
    # (bounds' masks=None without drafted rows: every row sees the cache alone)
    most = ref.bounds(*got, H, 112)
    assert bool(((O.double() - O2.view_as(O).double()).abs().cpu() <= 2 * most["O"]).all())
    assert bool(((lse.double() - lse2.view_as(lse).double()).abs().cpu() <= 2 * most["lse"]).all())


@pytest.mark.parametrize("rows", [1, 6, 70])
def test_shares_of_a_text(rows):
    """The pages of a text on two devices, the drafted rows on one of them: their partials merge to what one call gives."""
    x = _problem(2, "e4m3", 96, 2, 2, rows, [700, 260, 0], 16)
    (N, m, l, A, size), most = _expect(x)
    half = 17                                               # pages
    first = dict(x, lens=x["lens"].clamp(max=16 * half))
    second = dict(x, table=x["table"][:, half:].contiguous(), lens=(x["lens"] - 16 * half).clamp(min=0), K=None, V=None)
    parts = [_call(first), _call(second)]
    shape = x["Q"].shape
    flat = [[p[0].view(-1, rows, 96) for p in parts]] + [[p[i].view(-1, rows) for p in parts] for i in (1, 2)]
    O, lse = a2d.fix(*flat)
    some = l > 0
    exact = torch.where(some.unsqueeze(-1), N / torch.where(some, l, torch.ones_like(l)).unsqueeze(-1), torch.zeros_like(N))
    assert bool(((O.view(shape).double().cpu() - exact).abs() <= most["O"]).all())
    got = lse.view(shape[:3]).double().cpu()
    assert torch.equal(got == -math.inf, ~some) and bool(((got - m - torch.log(l)).abs()[some] <= 2 * most["lse"][some]).all())


@pytest.mark.parametrize("fmt, H", [("bf16", 64), ("e4m3", 128), ("e2m1", 80)])
@pytest.mark.parametrize("group, rows", [(1, 1), (4, 5), (2, 40)])
def test_what_may_hold_anything(fmt, H, group, rows):
    """Tokens behind a sequence's last, rows that are no tokens, drafted rows that no row sees: NaN and infinities there change no bit."""
    x = _problem(4, fmt, H, 2, group, rows, [70, 33, 0, 16], 48)
    clean = _call(x, normalised=True), _call(x)
    values = ref.cache_values(x["cache"], 0)
    used = torch.zeros(values.shape[0], values.shape[2], dtype=torch.bool)
    for b, n in enumerate(x["lens"].tolist()):
        for t in range(n):
            used[int(x["table"][b, t // 48]), t % 48] = True
    at = (~used).unsqueeze(1).expand(-1, 2, -1).cuda()
    for i, c in enumerate(x["cache"]):
        raw = c.view(torch.uint8) if c.element_size() == 1 else c
        raw[at] = 255 if c.element_size() == 1 else [math.nan, math.inf][i]
    x["table"][1, 1:] = 10 ** 9                              # (entries of no tokens are not looked at)
    x["table"][2] = -5
    dead = (torch.tensor([[v == -2 for v in p] for p in x["parents"]])).cuda()
    for name, bad in (("Q", math.nan), ("K", math.inf), ("V", math.nan)):
        x[name] = x[name].clone()
        x[name].transpose(1, 2)[dead] = bad
    assert _same(clean[0], _call(x, normalised=True)) and _same(clean[1], _call(x))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("group, rows", [(1, 5), (4, 9), (3, 10), (2, 40)])
def test_values_that_are_not_finite(bad, group, rows):
    """A drafted row's V with a NaN or an infinity reaches the rows that see it, and no others; a key's NaN likewise."""
    x = _problem(6, "e4m3", 80, 2, group, rows, [50 if rows != 10 else 600, 0], 16)
    clean = [y.float() for y in _call(x, normalised=True)]
    seen = [ref.ancestors(p) for p in x["parents"]]
    hit = torch.tensor([[s is not None and 2 in s for s in b] for b in seen]).view(2, 1, rows, 1).cuda()
    v = dict(x, V=x["V"].clone())
    v["V"][:, 1, 2, 37] = bad
    O, lse = (y.float() for y in _call(v, normalised=True))
    column = torch.zeros(80, dtype=torch.bool, device="cuda")
    column[37] = True
    head = (torch.arange(2 * group, device="cuda") >= group).view(1, -1, 1, 1)
    want = hit & head & column
    assert torch.equal(lse, clean[1])
    assert torch.equal(torch.where(want, 0.0, O), torch.where(want, 0.0, clean[0]))
    got = O[want.expand_as(O)]
    assert bool((torch.isnan(got) if math.isnan(bad) else got == bad).all())
    k = dict(x, K=x["K"].clone())
    k["K"][:, 1, 2, 37] = math.nan
    O, lse = (y.float() for y in _call(k, normalised=True))
    want = (hit & head).expand_as(O)
    assert torch.equal(torch.isnan(O), want) and torch.equal(torch.where(want, 0.0, O), torch.where(want, 0.0, clean[0]))
    assert torch.equal(torch.isnan(lse), want[..., 0])


def test_pages_that_are_none():
    """Tokens of entries that name no page are not seen; all of a text's: the empty partial."""
    x = _problem(8, "e2m1", 64, 1, 2, 3, [200, 100, 64], 16, drafts=False, masked=False)
    x["table"][0, 3], x["table"][0, 12], x["table"][1, 0] = -1, x["cache"][0].shape[0], 2 ** 31 - 1
    x["table"][2] = -2 ** 31
    values = [ref.cache_values(x["cache"], i) for i in range(2)]
    got = ref.attention(x["Q"], values, x["table"], x["lens"], scale=x["scale"])
    _check(x, (got, ref.bounds(*got, 64, 203)))
    assert bool((_call(x)[1][2] == -math.inf).all())


def test_lengths_beyond():
    """Longer than the host's bound, than the table; negative."""
    x = _problem(9, "e4m3", 64, 2, 2, 2, [160, 160, 160], 16)
    want = dict(x, lens=torch.tensor([100, 0, 60], dtype=torch.int32))
    far = dict(x, lens=torch.tensor([2 ** 31 - 1, -2 ** 31, 60], dtype=torch.int32))
    assert _same(_call(want, max_tokens=100), _call(far, max_tokens=100))
    assert _same(_call(dict(x, lens=x["lens"])), _call(dict(x, lens=torch.full((3,), 2 ** 31 - 1, dtype=torch.int32))))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [1, 7, 40])
def test_views(fmt, rows):
    """Q, K, V and O as a model keeps them, numbers that begin anywhere: the bits of plain tensors."""
    x = _problem(10, fmt, 96, 2, 4, rows, [300, 77, 5], 48)
    want = _call(x, normalised=True)
    n = 3
    packed = torch.empty(n, rows, 12 + 2, 96, dtype=torch.bfloat16, device="cuda").fill_(math.nan)
    views = {}
    for name, at in (("Q", slice(1, 9)), ("K", slice(9, 11)), ("V", slice(11, 13))):
        views[name] = packed[:, :, at].permute(0, 2, 1, 3)
        views[name].copy_(x[name])
    odd = _offset
    out = torch.full((n, rows, 10, 96), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(n, 8, rows, device="cuda")
    got = a2d.partial_fwd_cached(views["Q"], x["cache"], odd(x["table"]), odd(x["lens"]), K=views["K"], V=views["V"], masks=odd(x["masks"]),
                                 scale=x["scale"], out=(out[:, :, 1:9].permute(0, 2, 1, 3), lse), normalised=True)
    assert _same(got, want) and bool((out[:, :, 0] == 7).all()) and bool((out[:, :, 9] == 7).all())


def _offset(t):
    """The tensor on the device, one element behind a multiple of 16 bytes."""
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    room[1:].copy_(t.flatten())
    return room[1:].view(t.shape)


@pytest.mark.parametrize("group, rows", [(4, 1), (1, 20), (2, 40)])
def test_walks_shared_and_not(group, rows):
    """Without memory for parts (the C boundary without a workspace) one workgroup walks a text: the same within the bounds; with it, the
    same bits each time."""
    x = _problem(12, "e4m3", 128, 2, group, rows, [4000, 31, 0, 900], 64)
    want = _expect(x)
    a, b = _call(x), _call(x)
    assert _same(a, b)
    _check(x, want)
    K, V, Ks, Vs = x["cache"]
    table, lens, masks = x["table"].cuda(), x["lens"].cuda(), x["masks"].cuda()
    c = a2d.CacheDesc(a2d.CACHE_E4M3, 2, 128, 64, K.shape[0], 4, table.shape[1], 0, K.data_ptr(), V.data_ptr(), Ks.data_ptr(), Vs.data_ptr(),
                      table.data_ptr())
    d = a2d.CachedDesc(heads=2 * group, rows=rows, max_tokens=0, scale=x["scale"], lens=lens.data_ptr(), masks=masks.data_ptr())
    need = a2d.lib().a2d_cached_workspace_bytes(ctypes.byref(c), ctypes.byref(d))
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    N, m, l = (torch.empty_like(t) for t in a)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    call = lambda ws, bytes: a2d.lib().a2d_partial_fwd_cached(ctypes.byref(c), ctypes.byref(d), 0, ptr(x["Q"]), ptr(x["K"]), ptr(x["V"]), ptr(N),
                                                               ptr(m), ptr(l), ws, bytes, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert call(ptr(ws), need - 1) == -4 and b"workspace" in a2d.lib().a2d_last_error()
    assert call(ptr(ws), need) == 0
    assert _same((N, m, l), a)
    assert call(None, 0) == 0
    (N0, m0, l0, A, size), most = want
    some = l0 > 0
    assert torch.equal((l == 0).cpu(), ~some)
    f = torch.where(some, torch.exp(m.double().cpu() - m0), torch.ones_like(m0)).unsqueeze(-1)
    assert bool(((N.double().cpu() * f - N0).abs() <= most["N"] + most["m"].unsqueeze(-1) * A)[some].all())


def test_two_streams_at_once():
    xs = [_problem(20 + i, "e4m3", 128, 4, 2, 3, [3000, 500, 1], 64) for i in range(2)]
    args = [(x["Q"], x["cache"], x["table"].cuda(), x["lens"].cuda(), x["K"], x["V"], x["masks"].cuda()) for x in xs]
    want = [a2d.partial_fwd_cached(*a, normalised=True) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(a2d.partial_fwd_cached(*args[i], normalised=True))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(_same(g, want[i]) for g in got[i])


@pytest.mark.parametrize("rows", [1, 9, 40])
def test_a_step_as_a_graph(rows):
    """Tree, attention and the write of the kept rows captured and replayed, with new lengths, tables and rows between the replays and other
    calls of the library beside them: each replay gives what calls give."""
    fmt, H, page_rows, columns, n = "e4m3", 128, 32, 40, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = _problem(30, fmt, H, 2, 2, rows, [1200, 1, 40], page_rows, masked=False)
    held = {"Q": x["Q"], "K": x["K"], "V": x["V"], "table": x["table"].cuda(), "lens": x["lens"].cuda(), "cache": x["cache"],
            "parents": torch.full((n, rows), -1, dtype=torch.int32, device="cuda"), "index": torch.zeros(n, rows, dtype=torch.int32, device="cuda")}

    def step(h):
        masks, positions = a2d.tree_masks(h["parents"], h["lens"])
        O, lse = a2d.partial_fwd_cached(h["Q"], h["cache"], h["table"], h["lens"], h["K"], h["V"], masks, max_tokens=1200, normalised=True)
        a2d.cache_write(h["cache"], h["table"], h["K"], h["V"], h["lens"], index=h["index"])
        return [O, lse, masks, positions, *(c.view(torch.uint8) for c in h["cache"])]

    copy = lambda h: {k: tuple(c.clone() for c in v) if k == "cache" else v.clone() for k, v in h.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(copy(held))
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        mine = copy(held)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(mine)
        graphs.append((g, mine, out))
    for turn in range(4):
        for g, mine, out in graphs:
            mine["lens"].copy_(torch.randint(0, 1200, (n,), generator=gen, device="cuda"))
            mine["Q"].copy_(torch.randn(mine["Q"].shape, generator=gen, device="cuda"))
            mine["K"].copy_(torch.randn(mine["K"].shape, generator=gen, device="cuda"))
            mine["parents"].copy_(torch.randint(-1, 3, (n, rows), generator=gen, device="cuda"))
            mine["index"].copy_(torch.randint(-1, rows, (n, rows), generator=gen, device="cuda"))
            want = [y.clone() for y in step(copy(mine))]
            torch.cuda.synchronize()
            g.replay()
            _call(x)                                        # (eager, beside it)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_a_foreign_capture_takes_no_memory():
    """A stream captured by the program itself: the call shares no walks there, and numbers that it would have to copy are refused."""
    x = _problem(31, "e4m3", 128, 2, 2, 5, [3000, 400], 64)
    table, lens, masks = x["table"].cuda(), x["lens"].cuda(), x["masks"].cuda()
    out = [torch.empty_like(t) for t in _call(x)]
    call = lambda lens: a2d.partial_fwd_cached(x["Q"], x["cache"], table, lens, x["K"], x["V"], masks, scale=x["scale"], out=out)
    hip = ctypes.CDLL(a2d._loaded_hip_runtime())
    side, graph, run = torch.cuda.Stream(), ctypes.c_void_p(), ctypes.c_void_p()
    stream, odd = ctypes.c_void_p(side.cuda_stream), _offset(lens)
    with torch.cuda.stream(side):
        call(lens)                                          # (kernels loaded)
        torch.cuda.synchronize()
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        assert hip.hipStreamBeginCapture(stream, ctypes.c_int(1)) == 0       # hipStreamCaptureModeThreadLocal
        try:
            call(lens)
            with pytest.raises(a2d.A2DError):
                call(odd)
        finally:
            ended = hip.hipStreamEndCapture(stream, ctypes.byref(graph))
        assert ended == 0 and torch.cuda.memory_stats()["allocation.all.allocated"] == before
    assert hip.hipGraphInstantiate(ctypes.byref(run), graph, None, None, ctypes.c_size_t(0)) == 0
    (N, m, l, A, size), most = _expect(x)
    first = None
    for _ in range(3):
        for t in out:
            t.fill_(math.nan)
        torch.cuda.synchronize()
        assert hip.hipGraphLaunch(run, stream) == 0
        torch.cuda.synchronize()
        some = l > 0
        f = torch.where(some, torch.exp(out[1].double().cpu() - m), torch.ones_like(m)).unsqueeze(-1)
        assert bool(((out[0].double().cpu() * f - N).abs() <= most["N"] + most["m"].unsqueeze(-1) * A)[some].all())
        assert torch.equal((out[2] == 0).cpu(), ~some)
        first = first or [t.clone() for t in out]
        assert _same(first, out)
    assert hip.hipGraphExecDestroy(run) == 0 and hip.hipGraphDestroy(graph) == 0


def test_a_cache_of_more_than_4_gib():
    """Offsets in codes that pass 32 bits (5.4 GiB of K, pages at its ends)."""
    kv_heads, page_rows, H, pages = 8, 64, 128, 88000
    cache = a2d.cache_empty(pages, kv_heads, page_rows, H)
    table = torch.tensor([[pages - 1, 0, pages - 2], [65535, 65536, 70000]], dtype=torch.int32)
    lens = torch.tensor([150, 192], dtype=torch.int32)
    gen = torch.Generator(device="cuda").manual_seed(5)
    K, V = (torch.randn(2, kv_heads, 192, H, generator=gen, device="cuda") for _ in range(2))
    a2d.cache_write(cache, table.cuda(), K, V, torch.zeros(2, dtype=torch.int32, device="cuda"))
    back = a2d.cache_read(cache, table.cuda(), lens.cuda(), 192, out_dtype=torch.float32)
    small = a2d.cache_empty(6, kv_heads, page_rows, H)
    near = torch.arange(6, dtype=torch.int32).view(2, 3)
    a2d.cache_write(small, near.cuda(), K, V, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert _same(back, a2d.cache_read(small, near.cuda(), lens.cuda(), 192, out_dtype=torch.float32))
    for rows in (1, 70):
        Q = torch.randn(2, 8, rows, H, generator=gen, device="cuda").bfloat16()
        k, v = (torch.randn(2, kv_heads, rows, H, generator=gen, device="cuda").bfloat16() for _ in range(2))
        assert _same(a2d.partial_fwd_cached(Q, cache, table.cuda(), lens.cuda(), k, v), a2d.partial_fwd_cached(Q, small, near.cuda(), lens.cuda(), k, v))


def test_many_sequences():
    """More than the 64 whose lengths a wavefront looks at together, none among them; one key/value head."""
    lens = [(37 * i) % 200 if i % 5 else 0 for i in range(150)]
    lens[70], lens[149] = 1500, 900
    _check(_problem(13, "e4m3", 64, 1, 2, 2, lens, 16), max_tokens=1500)
    _check(_problem(14, "bf16", 64, 1, 1, 1, lens, 16, masked=False, drafts=False), _without_drafts(14, lens), max_tokens=1500)


def test_hundreds_of_sequences():
    """More than the 256 whose lengths are asked for at once."""
    lens = [(13 * i) % 40 if i % 3 else 0 for i in range(600)]
    lens[3], lens[255], lens[256], lens[599] = 700, 100, 650, 300
    _check(_problem(21, "e4m3", 64, 1, 1, 2, lens, 16), max_tokens=700)


def _without_drafts(seed, lens):
    x = _problem(seed, "bf16", 64, 1, 1, 1, lens, 16, masked=False, drafts=False)
    values = [ref.cache_values(x["cache"], i) for i in range(2)]
    got = ref.attention(x["Q"], values, x["table"], x["lens"], scale=x["scale"])
    return got, ref.bounds(*got, 64, max(lens))


@pytest.mark.parametrize("rows, group", [(300, 1), (1, 1), (33, 1), (513, 1)])
def test_chains_of_any_length(rows, group):
    """A chunk of a prompt over what is cached of it."""
    _check(_problem(15, "e4m3", 64, 1, group, rows, [100, 0], 16, masked=False))


@pytest.mark.parametrize("sigma", [8.0, 1e-3])
def test_peaks_and_flat_rows(sigma):
    _check(_problem(16, "bf16", 128, 1, 4, 5, [1000, 300], 16, sigma=sigma))
    _check(_problem(17, "e4m3", 128, 1, 4, 40, [1000, 300], 16, sigma=sigma))


def test_one_page_of_odd_size_for_each_sequence():
    """A contiguous cache is one page for each sequence."""
    _check(_problem(18, "e2m1", 96, 2, 2, 4, [1007, 513], 1008, extra=0))


def test_other_devices_and_types_are_refused():
    x = _problem(19, "e4m3", 64, 1, 1, 1, [16], 16)
    for wrong in (dict(Q=x["Q"].float()), dict(K=x["K"].float()), dict(V=None), dict(Q=x["Q"][..., :32]), dict(K=x["K"].expand(2, -1, -1, -1)),
                  dict(Q=x["Q"].expand(-1, 3, -1, -1)[:, :, :, :]), dict(masks=x["masks"].int()), dict(masks=x["masks"][0]),
                  dict(lens=x["lens"].long()), dict(table=x["table"].long()), dict(cache=x["cache"][:2]), dict(cache=x["cache"][::-1]),
                  dict(cache=(x["cache"][0].view(torch.int8),) + x["cache"][1:])):
        with pytest.raises(a2d.A2DError):
            _call(dict(x, **wrong))
    out = [torch.empty(1, 1, 1, 64, device="cuda"), torch.empty(1, 1, 1, device="cuda"), torch.empty(1, 1, 1, device="cuda")]
    assert _call(x, out=out)[0].data_ptr() == out[0].data_ptr()
    for i in range(3):
        bad = list(out)
        bad[i] = bad[i].double()
        with pytest.raises(a2d.A2DError):
            _call(x, out=bad)
    with pytest.raises(a2d.A2DError):
        _call(x, max_tokens=-1)
    with pytest.raises(a2d.A2DError):
        a2d.cache_write(x["cache"], x["table"].cuda(), x["K"].half(), x["V"].half(), x["lens"].cuda())
    with pytest.raises(a2d.A2DError):
        a2d.cache_read(x["cache"], x["table"].cuda(), x["lens"].cuda(), 4, out_dtype=torch.float16)
