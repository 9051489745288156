"""Chunks of a prompt - a chain of many rows - over what is cached of it, and the host's bound on the lengths, against 64 bits."""
import math

import pytest
import torch

from paper_2503_15758_amd import binding as a2d
from test_gpu_cached_attention import _call, _check, _expect, _problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt, H", [("bf16", 64), ("bf16", 128), ("e4m3", 80), ("e4m3", 128), ("e2m1", 96), ("e2m1", 64)])
@pytest.mark.parametrize("kv_heads, group, rows", [(2, 1, 150), (1, 4, 70), (2, 2, 257), (1, 3, 400)])
def test_chunks(fmt, H, kv_heads, group, rows):
    """Blocks that begin in the middle of a head's rows, several query heads in one block, drafted steps that a block skips."""
    _check(_problem(30, fmt, H, kv_heads, group, rows, [100, 0, 700], 48, masked=False))


def test_a_prompt_in_chunks():
    """Written chunk by chunk, each chunk's rows seen by themselves: what the whole prompt in one chunk gives."""
    gen = torch.Generator().manual_seed(1)
    heads, kv_heads, H, n = 4, 2, 64, 500
    Q, K, V = (torch.randn(1, h, n, H, generator=gen).bfloat16().cuda() for h in (heads, kv_heads, kv_heads))
    cache = a2d.cache_empty(32, kv_heads, 16, H, a2d.CACHE_BF16)
    table = torch.randperm(32, generator=gen).view(1, 32).int().cuda()
    length = lambda t: torch.tensor([t], dtype=torch.int32, device="cuda")
    O, lse = [], []
    for at, rows in ((0, 1), (1, 200), (201, 33), (234, 266)):
        q, k, v = (x[:, :, at:at + rows] for x in (Q, K, V))
        o, s = a2d.partial_fwd_cached(q, cache, table, length(at), k, v, max_tokens=at, normalised=True)
        a2d.cache_write(cache, table, k, v, length(at))
        O.append(o)
        lse.append(s)
    x = {"cache": cache, "table": table.cpu(), "lens": torch.tensor([0], dtype=torch.int32), "Q": Q, "K": K, "V": V, "masks": None, "scale": 1 / math.sqrt(H)}
    (N, m, l, A, size), most = _expect(x)
    exact = N / l.unsqueeze(-1)
    assert bool(((torch.cat(O, 2).double().cpu() - exact).abs() <= most["O"]).all())
    assert bool(((torch.cat(lse, 2).double().cpu() - m - torch.log(l)).abs() <= most["lse"]).all())


@pytest.mark.parametrize("bound", [700, 701, 1 << 30, 0])
@pytest.mark.parametrize("rows", [1, 9, 40])
def test_the_hosts_bound_is_in_tokens(rows, bound):
    x = _problem(31, "e4m3", 64, 2, 2, rows, [700, 33, 0, 100], 16)
    _check(x, max_tokens=bound)
    if rows > 1:
        return
    short = dict(x, lens=x["lens"].clamp(max=24))           # (a bound in pages, say, cuts the lengths)
    for a, b in zip(_call(x, max_tokens=24), _call(short, max_tokens=24)):
        assert torch.equal(a, b)
