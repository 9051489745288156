"""Rotary positions with several axes against 64 bits.  Bounds: an angle is off by 2^-32 turns and the sine and cosine by 2^-18 (16-bit
results: the hardware's) or 4 half steps of fp32; two products and a sum of fp32; the result's own rounding."""
import math

import pytest
import torch

from scored_reference import half_step

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def a2d():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding
    binding.lib()
    return binding


def turned(x, positions, freqs, axis, interleaved, inverse):
    """(result, size of what it is made of) in 64 bits"""
    x, pos = x.detach().cpu().double(), positions.cpu().double()
    pos = pos.unsqueeze(0) if pos.dim() == 2 else pos
    pos = pos.repeat_interleave(x.shape[0] // pos.shape[0], 0)
    out, size = x.clone(), torch.zeros_like(x)
    for p in range(freqs.numel()):
        phi = pos[:, int(axis[p])] * float(freqs[p]) * (-1 if inverse else 1)
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + x.shape[2] // 2)
        out[..., i] = x[..., i] * torch.cos(phi) - x[..., j] * torch.sin(phi)
        out[..., j] = x[..., i] * torch.sin(phi) + x[..., j] * torch.cos(phi)
        size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return out, size


def check(got, want, size, out_dtype, what, far=0.0):
    got, r = got.detach().cpu().double(), half_step(out_dtype)
    e = (2.0 ** -18 if r else 4 * U) + 2 * math.pi * 2.0 ** -32 + far
    bound = (size * (e + 3 * U)) * (1 + r) + (r or U) * want.abs()
    bad = ((got - want).abs() > bound) | torch.isnan(got)
    assert not bad.any(), "%s: off %.3g" % (what, (got - want).abs().max().item())


def positions_of(sets, axes, rows, most, gen):
    p = torch.randint(-most if most > 100 else 0, most, (sets, axes, rows), generator=gen, dtype=torch.int32)
    return (p if sets > 1 else p[0]).contiguous().cuda()


# heads of Q and K, sets, rows, H, sections, type in, type out, most position
CASES = [(4, 2, 1, 50, 128, (16, 24, 24), "bf16", "bf16", 5000), (3, 1, 1, 1, 64, (32,), "bf16", "bf16", 10),
         (8, 4, 4, 1, 128, (16, 24, 24), "bf16", "bf16", 100000), (6, 6, 3, 37, 96, (10, 14), "f32", "bf16", 3000),
         (2, 2, 1, 333, 80, (20, 20), "f32", "f32", 50), (40, 8, 1, 777, 128, (64,), "bf16", "bf16", 1000000),
         (2, 2, 2, 9, 16, (3, 1, 2), "f32", "f32", 2000000000), (1, 1, 1, 70, 256, (1, 2, 3, 4, 5, 6, 7, 100), "bf16", "bf16", 7)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%d_%d_sets%d_rows%d_H%d_%s_%s" % (c[0], c[1], c[2], c[3], c[4], c[6], c[7]))
def test_rotary(a2d, case, interleaved):
    hq, hk, sets, rows, H, sections, ti, to, most = case
    print("rotary", case, interleaved, flush=True)
    gen = torch.Generator().manual_seed(5)
    Q, K = (torch.randn(h, rows, H, generator=gen).to(DT[ti]).cuda() for h in (hq, hk))
    pos = positions_of(sets, len(sections), rows, most, gen)
    freqs, axis = a2d.rotary_frequencies(H, sections)
    for inverse in (False, True):
        got = a2d.rotary((Q, K), pos, freqs, axis, interleaved=interleaved, inverse=inverse, out_dtype=DT[to])
        for x, y, name in zip((Q, K), got, "QK"):
            want, size = turned(x, pos, freqs, axis, interleaved, inverse)
            # (the reference's angle: 2^-52 of a large product)
            check(y, want, size, DT[to], name, far=2.0 ** -51 * most)
        alone = a2d.rotary(K, pos, freqs, axis, interleaved=interleaved, inverse=inverse, out_dtype=DT[to])
        assert torch.equal(alone, got[1])
    rest = torch.ones(H, dtype=torch.bool)                       # columns of no pair: as they were
    for p in range(sum(sections)):
        rest[[2 * p, 2 * p + 1] if interleaved else [p, p + H // 2]] = False
    assert torch.equal(got[0][..., rest.cuda()], Q[..., rest.cuda()].to(DT[to]))


def test_in_place_through_a_packed_projection(a2d):
    """Q and K of one [rows][3][heads][H] projection, turned where they lie; V, and the other columns of memory, stay."""
    rows, heads, H = 65, 4, 128
    gen = torch.Generator().manual_seed(6)
    qkv = torch.randn(rows, 3, heads, H, generator=gen).to(torch.bfloat16).cuda()
    Q, K = qkv[:, 0].permute(1, 0, 2), qkv[:, 1].permute(1, 0, 2)
    pos = positions_of(1, 3, rows, 900, gen)
    freqs, axis = a2d.rotary_frequencies(H, (16, 24, 24))
    apart = a2d.rotary((Q, K), pos, freqs, axis)
    before = qkv.clone()
    back = a2d.rotary((Q, K), pos, freqs, axis, out=(Q, K))
    assert back[0].data_ptr() == Q.data_ptr()
    assert torch.equal(Q, apart[0]) and torch.equal(K, apart[1]) and torch.equal(qkv[:, 2], before[:, 2])
    a2d.rotary(Q, pos, freqs, axis, inverse=True, out=Q)
    # (turned there and back: two roundings of a vector whose size stays)
    assert (Q.float() - before[:, 0].permute(1, 0, 2).float()).abs().max().item() <= 2 * 2.0 ** -8 * before[:, 0].abs().max().item() * math.sqrt(2)


def test_infinities_stay_where_no_pair_is(a2d):
    gen = torch.Generator().manual_seed(7)
    X = torch.randn(2, 3, 64, generator=gen).cuda()
    X[:, :, 60] = float("inf")                                   # (the partner of column 28, in no pair)
    freqs, axis = a2d.rotary_frequencies(64, (10, 10))
    got = a2d.rotary(X, positions_of(1, 2, 3, 9, gen), freqs, axis)
    assert torch.equal(got[:, :, 60], X[:, :, 60]) and torch.equal(got[:, :, 28], X[:, :, 28]) and not torch.isnan(got).any()


def test_gradient_is_the_inverse(a2d):
    """<turned(x), g> = <x, turned back(g)>: what a gradient is, of a linear map, in fp32."""
    gen = torch.Generator().manual_seed(8)
    x, g = (torch.randn(4, 100, 96, generator=gen).cuda() for _ in range(2))
    pos = positions_of(1, 2, 100, 5000, gen)
    freqs, axis = a2d.rotary_frequencies(96, (20, 28), restart=True)
    a = (a2d.rotary(x, pos, freqs, axis).double() * g.double()).sum().item()
    b = (x.double() * a2d.rotary(g, pos, freqs, axis, inverse=True).double()).sum().item()
    # (each element of either is off by 8 half steps of |x| + |its partner|)
    assert abs(a - b) <= 2 * 8 * U * 2 * (x.double().norm() * g.double().norm()).item()


def test_replayed(a2d):
    gen = torch.Generator().manual_seed(9)
    X = torch.randn(8, 40, 128, generator=gen).to(torch.bfloat16).cuda()
    pos = positions_of(1, 3, 40, 900, gen)
    freqs, axis = a2d.rotary_frequencies(128, (16, 24, 24))
    a2d.rotary(X, pos, freqs, axis)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = a2d.rotary(X, pos, freqs, axis)
    for i in range(3):
        pos.add_(17)
        eager = a2d.rotary(X, pos, freqs, axis)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, eager), i
