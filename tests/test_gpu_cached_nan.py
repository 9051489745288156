"""Scores that are NaN - a NaN in Q, in a drafted row's K, in a cached key -: every row that sees one is NaN in all that comes out of it, also where it
sees nothing else, and however its walk is shared; no other row changes a bit."""
import math

import pytest
import torch

import cached_reference as ref
from cached_calls import without_workspace
from paper_2503_15758_amd import binding as a2d
from test_gpu_cached_attention import _call, _problem, kernels  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# rows of a key/value head: 1, 3 (one row tile), 20 (two, over long texts), 80 and 160 (workgroups of 128 and 256)
FORMS = [(1, 1), (1, 3), (4, 5), (2, 40), (2, 80)]


def _outputs(x, **more):
    """(O, lse), (N, m, l), with walks shared and not."""
    for normalised in (True, False):
        yield _call(x, normalised=normalised, **more)
        yield without_workspace(x, normalised, **more)


def _hits(clean, bad, hit, **more):
    """hit [sequence][head][row]: the rows that see a NaN."""
    assert bool(hit.any()) and not bool(hit.all())
    for before, after in zip(_outputs(clean, **more), _outputs(bad, **more)):
        for i, (a, b) in enumerate(zip(before, after)):
            want = (hit.unsqueeze(-1) if i == 0 else hit).expand_as(b).to(b.device)
            assert torch.equal(torch.isnan(b), want), (len(before), i)
            assert torch.equal(torch.where(want, 0.0, b.float()), torch.where(want, 0.0, a.float())), (len(before), i)


def _bad_keys(x, tokens, head=0):
    """The problem with a NaN in head `head`'s K of tokens[b] (a list) of each sequence."""
    cache = [c.clone() for c in x["cache"]]
    rows = cache[0].shape[2]
    for b, some in enumerate(tokens):
        for t in some:
            page = int(x["table"][b, t // rows])
            if len(cache) == 2:
                cache[0][page, head, t % rows, 40] = math.nan
            else:
                cache[2][page, head, t % rows, 1] = 255
    return dict(x, cache=tuple(cache))


@pytest.mark.parametrize("fmt, H", [("bf16", 128), ("e4m3", 64), ("e2m1", 80)])
@pytest.mark.parametrize("group, rows", FORMS)
def test_a_query(kernels, fmt, H, group, rows):
    x = _problem(3, fmt, H, 2, group, rows, [2100, 70, 0, 33], 48)
    bad = dict(x, Q=x["Q"].clone())
    hit = torch.zeros(4, 2 * group, rows, dtype=torch.bool)
    for b, head in ((0, 0), (2, 2 * group - 1), (3, group)):
        bad["Q"][b, head, 0, 17] = math.nan
        hit[b, head, 0] = True
    _hits(x, bad, hit)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("group, rows", [(1, 3), (4, 5), (2, 40), (2, 80)])
def test_a_lone_drafted_key(kernels, fmt, group, rows):
    """Rows that follow the text, which is empty in one sequence: each sees itself alone there."""
    x = _problem(4, fmt, 96, 2, group, rows, [0, 70], 16)
    alone = torch.zeros(2, rows, (rows + 63) // 64, dtype=torch.int64)
    for i in range(rows):
        bit = 1 << (i % 64)
        alone[:, i, i // 64] = bit - (1 << 64) if bit >> 63 else bit
    x["masks"] = alone
    bad = dict(x, K=x["K"].clone())
    hit = torch.zeros(2, 2 * group, rows, dtype=torch.bool)
    for i in (0, rows - 1):
        bad["K"][:, 1, i, 50] = math.nan
        hit[:, group:, i] = True
    _hits(x, bad, hit)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("group, rows, step", [(1, 1, 32), (4, 5, 32), (2, 40, 64), (2, 80, 64)])
def test_the_last_key_of_a_walk(kernels, fmt, group, rows, step):
    """The last token of every other sequence, alone in its step; wherever the line of walks is cut, some of these steps are a run's only one."""
    n = 60
    lens = [step * (1 + 7 * b % 6) + 1 for b in range(n)]
    lens[7] = 1500
    x = _problem(5, fmt, 64, 1, group, rows, [1] * n, 16, masked=False, drafts=False, extra=20)
    # (pages that the sequences share, but for each one's last)
    x["table"] = torch.randint(n, n + 20, (n, 94), generator=torch.Generator().manual_seed(1)).int()
    for b, t in enumerate(lens):
        x["table"][b, (t - 1) // 16] = b
    x["lens"] = torch.tensor(lens, dtype=torch.int32)
    bad = _bad_keys(x, [[t - 1] if b % 2 else [] for b, t in enumerate(lens)])
    hit = (torch.arange(n) % 2 == 1).view(-1, 1, 1).expand(-1, group, rows)
    _hits(x, bad, hit)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("group, rows", FORMS)
def test_runs_of_keys(kernels, fmt, group, rows):
    """The first 128 tokens, the middle of a walk that many workgroups share, its end: whole steps and whole runs of nothing else."""
    lens = [2100, 2100, 2100, 300]
    x = _problem(6, fmt, 64, 2, group, rows, lens, 64)
    bad = _bad_keys(x, [range(128), range(700, 1400), range(1900, 2100), []], head=1)
    hit = torch.zeros(4, 2 * group, rows, dtype=torch.bool)
    hit[:3, group:] = (x["masks"] != 0).any(-1)[:3].unsqueeze(1)      # (rows that are no tokens see nothing)
    _hits(x, bad, hit)


@pytest.mark.parametrize("group, rows", FORMS)
def test_a_share_that_is_nan_is_not_left_out(group, rows):
    """Merged with the finite partial of another share of the text."""
    x = _problem(7, "e4m3", 64, 1, group, rows, [160], 16, drafts=False, masked=False)
    bad = _bad_keys(x, [range(160)])
    parts = [[t.view(-1, *t.shape[2:]) for t in _call(y)] for y in (x, bad)]
    for first, second in (parts, parts[::-1]):
        O, _ = a2d.fix(*([a, b] for a, b in zip(first, second)))
        assert bool(torch.isnan(O).all())


@pytest.mark.parametrize("group, rows", FORMS)
def test_infinite_scores(kernels, group, rows):
    """A key with an infinity: NaN to the rows whose score it makes infinite, of weight 0 to those where it is -inf, to which a lone one is nothing."""
    x = _problem(8, "bf16", 64, 1, group, rows, [1000, 1], 16, drafts=False, masked=False)
    for b, t in ((0, 500), (1, 0)):
        x["cache"][0][int(x["table"][b, t // 16]), 0, t % 16, 40] = math.inf
    up = torch.rand(2, group, rows, generator=torch.Generator().manual_seed(1)) < 0.5
    x["Q"][..., 40] = torch.where(up, 1.0, -1.0).bfloat16().cuda()
    got = ref.attention(x["Q"], [ref.cache_values(x["cache"], i) for i in range(2)], x["table"], x["lens"], scale=x["scale"])
    N, m, l, A, size = got
    most = ref.bounds(N, m, l, A, torch.where(torch.isinf(size), 100.0, size), 64, 1000)          # (the finite keys': below 100)
    down = ~up[0]
    for call in (_call, without_workspace):
        n, top, sum_ = (y.double().cpu() for y in call(x))
        assert all(bool(torch.isnan(y[up]).all()) and not bool(torch.isnan(y[~up]).any()) for y in (n, top, sum_))
        assert bool((sum_[1][~up[1]] == 0).all()) and bool((n[1][~up[1]] == 0).all()) and bool((top[1][~up[1]] == -math.inf).all())
        f = torch.exp(top - m)[0]
        assert bool(((sum_[0] * f - l[0]).abs() <= most["l"][0] + most["m"][0] * l[0])[down].all())
        off = (n[0] * f.unsqueeze(-1) - N[0]).abs()
        assert bool((off <= most["N"][0] + most["m"][0].unsqueeze(-1) * A[0])[down].all())
        O, lse = (y.float().cpu() for y in call(x, normalised=True))
        assert torch.equal(torch.isnan(O), up.unsqueeze(-1).expand_as(O)) and torch.equal(torch.isnan(lse), up)
        assert bool((lse[1][~up[1]] == -math.inf).all())
