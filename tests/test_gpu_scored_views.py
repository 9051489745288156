"""Calls under score rules and rotary calls on views that begin anywhere, on part of a head, and without memory for partial results.
Bounds: tests/scored_reference.py."""
import ctypes

import pytest
import torch

from scored_reference import Scored, within
from test_gpu_rotary import check, turned
from test_gpu_scored import check_fwd, inputs, int32, slopes_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def a2d():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding
    binding.lib()
    return binding


def from_(x, n):
    """x as a view that begins n numbers behind a multiple of 16 bytes"""
    y = torch.zeros(x.numel() + n, dtype=x.dtype, device="cuda")[n:].view(x.shape)
    assert y.copy_(x).is_contiguous() and y.data_ptr() % 16 == (n * x.element_size()) % 16
    return y


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rules_that_begin_anywhere(a2d, dt):
    """A rank's slopes of all heads', a chunk's ranges, the starts and prefixes behind the first, positions behind other axes': as if
    they stood at the front, also replayed, when they have changed since."""
    heads, nq = 4, 70
    Q, K, V, dO = inputs(heads, 2, nq, 90, 64, dt)
    starts, prefix = int32([0, 20, 21, 85]), int32([5, 0, 9])
    ranges, slopes = a2d.document_ranges(starts, nq, prefix, first=3), slopes_of(heads)
    pos = torch.arange(2 * nq, dtype=torch.int32, device="cuda").view(2, nq)
    freqs, axis = a2d.rotary_frequencies(64, (16, 16))
    O, lse = a2d.partial_fwd_scored(Q, K, V, slopes=slopes, ranges=ranges, normalised=True)

    def run(slopes, ranges, starts, prefix, pos):
        return (a2d.document_ranges(starts, nq, prefix, first=3), a2d.rotary(Q, pos, freqs, axis),
                *a2d.partial_fwd_scored(Q, K, V, slopes=slopes, ranges=ranges, normalised=True),
                *a2d.partial_bwd_scored(Q, K, V, O, dO, lse, slopes=slopes, ranges=ranges))

    given = (slopes, ranges, starts, prefix, pos)
    want = run(*given)
    for n in (1, 2, 3):
        views = tuple(from_(x, n) for x in given)
        got = run(*views)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(*views)
    for i in range(3):
        views[0].mul_(0.5)
        views[4].add_(3)
        eager = run(views[0].clone(), ranges, starts, prefix, views[4].clone())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, eager)), i


def test_rotary_on_part_of_a_head(a2d):
    """The first r of H columns turned in place, through a view: pairs (p, p + r / 2), frequencies over r; the others stay."""
    heads, rows, H, r = 3, 40, 128, 32
    gen = torch.Generator().manual_seed(3)
    X = torch.randn(heads, rows, H, generator=gen).to(torch.bfloat16).cuda()
    before, pos = X.clone(), torch.arange(rows, dtype=torch.int32, device="cuda").view(1, rows)
    freqs, axis = a2d.rotary_frequencies(r, (r // 2,))
    assert freqs.tolist() == [10000.0 ** (-2.0 * p / r) for p in range(r // 2)]
    a2d.rotary(X[..., :r], pos, freqs, axis, out=X[..., :r])
    check(X[..., :r], *turned(before[..., :r], pos, freqs, axis, False, False), X.dtype, "turned")
    assert torch.equal(X[..., r:], before[..., r:])


# heads, kv_heads, nq, nkv, H: with memory in parts - of 128 rows in two key lanes, in workgroups of four wavefronts, of 32 rows
SHAPES = [(40, 8, 200, 1300, 128), (1, 1, 129, 1300, 96), (2, 1, 130, 1000, 80), (32, 8, 1, 1133, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%dx%dx%d_H%d" % s)
def test_without_memory(a2d, shape):
    """The C boundary has no memory for parts: whole walks, P rounded as with it."""
    heads, kvh, nq, nkv, H = shape
    Q, K, V, _ = inputs(heads, kvh, nq, nkv, H, "bf16", sigma=3.0)
    ref = Scored(Q, K, V, softcap=20.0).partial()
    out = tuple(torch.full(s, float("nan"), device="cuda") for s in ((heads, nq, H), (heads, nq), (heads, nq)))
    d, r = a2d.tile_desc(Q, K, 0, 0, False, H ** -0.5), a2d.ScoreRules(softcap=20.0, token_step=1, range_sets=1)
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    assert a2d.lib().a2d_partial_fwd_scored(ctypes.byref(d), kvh, ctypes.byref(r), 0, p(Q), p(K), p(V), *map(p, out), None, 0,
                                            ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    check_fwd(out, ref, False, Q.dtype, "without memory")
    fine = a2d.scored_route(heads, nq, nkv, H, kv_heads=kvh, softcap=20.0)["fine"]
    a, b = (x[0] / x[2].unsqueeze(2) for x in (out, a2d.partial_fwd_scored(Q, K, V, softcap=20.0)))
    # (each probability is rounded anew where a part has a maximum of its own: by 2^-17 or 2^-8 of itself on either side; the fp32 sums and the
    # scores' 2^x beside them are 2^-17 too: nkv + 160 roundings, and 2^-24 of scores up to 20 log2(e), twice)
    step = (2.0 ** -17 if fine else 2.0 ** -8) + (nkv + 160 + 60) * 2.0 ** -24
    assert ((a - b).norm() / b.norm()).item() <= 2 * step


def test_a_batch_under_a_bias(a2d):
    """Caches that end together: each sequence's own distances.  Caches that begin together, asked from behind the longest: every bias of a
    shorter one is too large by the same tokens, O is right and lse lower by slope times them."""
    heads, kvh, H, lens = 4, 2, 64, [200, 77]
    Q, K, V, _ = inputs(2 * heads, 2 * kvh, 1, 200, H, "bf16")
    slopes = slopes_of(heads).repeat(2)
    ends = a2d.partial_fwd_scored(Q, K, V, q_off=199, slopes=slopes, ranges=int32([[[200 - n, 200]] for n in lens]), normalised=True)
    begins = a2d.partial_fwd_scored(Q, K, V, q_off=199, slopes=slopes, ranges=int32([[[0, n]] for n in lens]), normalised=True)
    for i, n in enumerate(lens):
        h, k = slice(i * heads, (i + 1) * heads), slice(i * kvh, (i + 1) * kvh)
        s = Scored(Q[h], K[k, 200 - n:], V[k, 200 - n:], q_off=n - 1, slopes=slopes[h]).partial()
        check_fwd((ends[0][h], ends[1][h]), s, True, Q.dtype, "ending together")
        s = Scored(Q[h], K[k, :n], V[k, :n], q_off=n - 1, slopes=slopes[h]).partial()
        s["lse"] = s["lse"] - slopes[h].cpu().double().unsqueeze(1) * (200 - n)
        # (the scores are rounded next to a bias that is larger by slope times up to 123 tokens)
        more = 32 * 2.0 ** -24 * slopes[h].max().item() * 200
        s["e_O"], s["e_lse"] = s["e_O"] + more * V[k].abs().max().item(), s["e_lse"] + more
        check_fwd((begins[0][h], begins[1][h]), s, True, Q.dtype, "beginning together")


# heads, kv_heads, rows, H, type, window
WINDOWS = [(4, 2, 1500, 128, "bf16", 200), (16, 16, 700, 64, "bf16", 64), (2, 1, 300, 80, "f32", 33), (6, 3, 150, 96, "bf16", 1)]


@pytest.mark.parametrize("case", WINDOWS, ids=lambda c: "%dx%dx%d_H%d_%s_window%d" % c)
def test_sliding_windows(a2d, case):
    """Each row sees the last `window` tokens up to itself: ranges that move by a token a row, under a cap, with a bias too."""
    heads, kvh, n, H, dt, window = case
    print("window", case, flush=True)
    Q, K, V, dO = inputs(heads, kvh, n, n, H, dt)
    t = torch.arange(n, dtype=torch.int32, device="cuda")
    ranges = torch.stack([(t - window + 1).clamp(min=0), t + 1], 1).contiguous()
    for rules in (dict(softcap=8.0), dict(softcap=8.0, slopes=slopes_of(heads))):
        s = Scored(Q, K, V, ranges=ranges, **rules)
        f = s.partial()
        check_fwd(a2d.partial_fwd_scored(Q, K, V, ranges=ranges, normalised=True, **rules), f, True, Q.dtype, "window")
        O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
        want = s.gradients(O, dO, lse)
        for x, name in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, ranges=ranges, **rules), ("dQ", "dK", "dV")):
            within(x, want[name], want["e_" + name], "window %s" % name)
        # (a range that begins in front of the first token, and the mask instead of its end, say the same)
        open_ = torch.stack([t - window + 1, torch.full_like(t, 2 ** 31 - 1)], 1).contiguous()
        a = a2d.partial_fwd_scored(Q, K, V, ranges=open_, causal=True, normalised=True, **rules)
        check_fwd(a, f, True, Q.dtype, "window")


@pytest.mark.parametrize("dt, rows", [("bf16", 333), ("bf16", 40), ("f32", 130)])
def test_a_batch_of_prompts(a2d, dt, rows):
    """Sequences of different lengths whose last rows are asked for at once, caches ending together: one of them shorter than the rows."""
    heads, kvh, H, lens, nkv = 4, 2, 64, [500, 90, 333], 500
    print("prompts", dt, rows, flush=True)
    Q, K, V, dO = inputs(3 * heads, 3 * kvh, rows, nkv, H, dt)
    first = nkv - rows
    ranges = torch.zeros(3, rows, 2, dtype=torch.int32)
    for b, n in enumerate(lens):
        for i in range(rows):
            ranges[b, i] = torch.tensor([nkv - n, first + i + 1])
    rules = dict(softcap=9.0, slopes=slopes_of(heads).repeat(3), ranges=ranges.cuda(), q_off=first)
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    got = a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules)
    check_fwd(got, f, True, Q.dtype, "prompts")
    assert rows < 90 or not got[0][heads: 2 * heads, : rows - 90].any()
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    want = s.gradients(O, dO, lse)
    for x, name in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules), ("dQ", "dK", "dV")):
        within(x, want[name], want["e_" + name], "prompts %s" % name)
