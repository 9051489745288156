"""Attention over the paged cache against 64 bits."""
import math

import pytest
import torch

import cached_reference as ref
from paper_2503_15758_amd import binding as a2d

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["matrix", "plain"])
def kernels(request):
    a2d.force_generic(request.param == "plain")
    yield request.param
    a2d.force_generic(False)


def _problem(seed, fmt, H, kv_heads, group, rows, lens, page_rows, masked=True, drafts=True, sigma=1.0, extra=2):
    gen = torch.Generator().manual_seed(seed)
    n, heads = len(lens), kv_heads * group
    columns = max(1, max(-(-max(v, 0) // page_rows) for v in lens))
    pages = n * columns + extra
    x = {"cache": ref.new_cache(gen, a2d, fmt, pages, kv_heads, page_rows, H, sigma), "scale": 1.0 / math.sqrt(H)}
    x["table"] = torch.randperm(pages, generator=gen)[:n * columns].view(n, columns).int()
    x["lens"] = torch.tensor(lens, dtype=torch.int32)
    x["Q"] = torch.randn(n, heads, rows, H, generator=gen).bfloat16().cuda()
    x["K"] = x["V"] = x["masks"] = None
    if drafts:
        x["K"], x["V"] = (sigma * torch.randn(n, kv_heads, rows, H, generator=gen).bfloat16().cuda() for _ in range(2))
    if masked:
        x["parents"] = [[-1] + [int(torch.randint(-1, i, (1,), generator=gen)) for i in range(1, rows)] for _ in range(n)]
        for p in x["parents"][1::2]:
            p[rows - (rows - 1) // 3:] = [-2] * ((rows - 1) // 3)
        words = [ref.mask_words(ref.ancestors(p), -(-rows // 64)) for p in x["parents"]]
        x["masks"] = torch.tensor(words, dtype=torch.int64)
    return x


def _call(x, **more):
    return a2d.partial_fwd_cached(x["Q"], x["cache"], x["table"].cuda(), x["lens"].cuda(), K=x["K"], V=x["V"],
                                  masks=None if x["masks"] is None else x["masks"].cuda(), scale=x["scale"], **more)


def _expect(x):
    values = [ref.cache_values(x["cache"], i) for i in range(2)]
    got = ref.attention(x["Q"], values, x["table"], x["lens"], x["K"], x["V"], x["masks"], x["scale"])
    keys = max(0, int(x["lens"].max())) + x["Q"].shape[2]
    n, heads, rows, H = x["Q"].shape
    return got, ref.bounds(*got, H, keys, coarse=heads // x["cache"][0].shape[1] * rows > 32)


def _check(x, want=None, **more):
    (N, m, l, A, size), most = want or _expect(x)
    some = l > 0
    O, lse = (y.double().cpu() for y in _call(x, normalised=True, **more))
    exact = torch.where(some.unsqueeze(-1), N / torch.where(some, l, torch.ones_like(l)).unsqueeze(-1), torch.zeros_like(N))
    assert bool(((O - exact).abs() <= most["O"]).all()), ((O - exact).abs() / most["O"]).max()
    L = m + torch.log(l)
    assert torch.equal(lse == -math.inf, ~some)
    assert bool(((lse - L).abs()[some] <= most["lse"][some]).all())
    n2, m2, l2 = (y.double().cpu() for y in _call(x, **more))
    assert torch.equal(m2 == -math.inf, ~some) and bool((l2[~some] == 0).all()) and bool((n2[~some] == 0).all())
    assert bool(((m2 - m).abs()[some] <= most["m"][some]).all())
    f = torch.where(some, torch.exp(m2 - m), torch.ones_like(m))       # (relative to the kernel's own m)
    assert bool(((l2 * f - l).abs()[some] <= (most["l"] + most["m"] * l)[some]).all())
    off = (n2 * f.unsqueeze(-1) - N).abs()
    assert bool((off[some] <= (most["N"] + most["m"].unsqueeze(-1) * A)[some]).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("H", [64, 80, 96, 128])
@pytest.mark.parametrize("kv_heads, group, rows", [(2, 1, 1), (1, 4, 1), (2, 2, 7), (1, 8, 3), (1, 3, 17), (1, 2, 70)])
def test_against_64_bits(kernels, fmt, H, kv_heads, group, rows):
    """Blocks of 16, 32 and 128 rows, one that is not full; lengths around the steps of 32 and the tiles of 16, none at all; odd pages."""
    _check(_problem(7, fmt, H, kv_heads, group, rows, [0, 1, 15, 48, 97, 300], 48))


@pytest.mark.parametrize("fmt, H", [("bf16", 64), ("e4m3", 128), ("e2m1", 80), ("e4m3", 96)])
@pytest.mark.parametrize("rows", [1, 5, 12, 40])
def test_long_and_short_together(fmt, H, rows):
    """Walks that many workgroups share beside ones of a step."""
    _check(_problem(11, fmt, H, 2, 2, rows, [5000, 1, 0, 31, 2049, 333], 16, masked=rows > 1), max_tokens=5000)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("H", [64, 80, 96, 128])
@pytest.mark.parametrize("group, rows, masked", [(1, 65, True), (2, 100, True), (8, 33, True), (1, 33, True), (3, 130, False), (1, 256, True)])
def test_many_rows(fmt, H, group, rows, masked):
    """Workgroups of 128 and 256 rows, several blocks, trees of more than a word, chains."""
    _check(_problem(5, fmt, H, 1, group, rows, [0, 65, 700], 48, masked=masked))
