"""Infinities in a cached V: a row that sees one has it in that column, as for a drafted row's V, in every format, form and sharing of the walk."""
import math

import pytest
import torch

from cached_calls import without_workspace
from test_gpu_cached_attention import _call, _problem, kernels  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def _with_values(x, tokens, columns):
    """Two problems: sequence b's tokens[b] with V of head 0 zero in the blocks of `columns`, and the same with numbers[i] in columns[i]."""
    both = []
    for numbers in (None, (math.inf, -math.inf, math.nan)):
        cache = [c.clone() for c in x["cache"]]
        rows = cache[1].shape[2]
        for b, some in enumerate(tokens):
            for t in some:
                page, row = int(x["table"][b, t // rows]), t % rows
                for i, c in enumerate(columns):
                    block = c // 32
                    if len(cache) == 2:
                        cache[1][page, 0, row, 32 * block:32 * block + 32] = 0
                        if numbers:
                            cache[1][page, 0, row, c] = numbers[i]
                        continue
                    bytes_ = cache[1].view(torch.uint8)[page, 0, row]
                    per = 1 if cache[1].dtype == torch.float8_e4m3fn else 2
                    bytes_[32 * block // per:32 * block // per + 32 // per] = 0
                    if not numbers:
                        continue
                    if math.isnan(numbers[i]):               # (a NaN takes its whole block)
                        cache[3][page, 0, row, block] = 255
                        continue
                    cache[3][page, 0, row, block] = 254     # 448 or 6 times 2^127
                    if per == 1:
                        bytes_[c] = 0x7E + (128 if numbers[i] < 0 else 0)
                    else:
                        bytes_[c // 2] = (7 + (8 if numbers[i] < 0 else 0)) << (4 * (c & 1))
        both.append(dict(x, cache=tuple(cache)))
    return both


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("H", [64, 80, 96, 128])
@pytest.mark.parametrize("group, rows", [(1, 1), (4, 5), (2, 40), (2, 80)])
def test_cached_values(kernels, fmt, H, group, rows):
    """In the first and in later steps, in the first and in later tiles of a step, in a tile that is not full."""
    x = _problem(2, fmt, H, 2, group, rows, [1001, 70, 100, 16], 48)
    tokens = [[0, 737], [65], [21, 99], []]
    columns = [3, H - 1] if H == 64 else [3, 33, H - 1]
    clean, bad = _with_values(x, tokens, columns)
    sees = torch.zeros(4, 2 * group, rows, dtype=torch.bool)
    sees[:3, :group] = (x["masks"] != 0).any(-1)[:3].unsqueeze(1)      # (rows that are no tokens see nothing)
    for normalised in (True, False):
        for call in (_call, without_workspace):
            before, after = call(clean, normalised=normalised), call(bad, normalised=normalised)
            for a, b in zip(before[1:], after[1:]):
                assert torch.equal(a, b)
            got, rest = after[0].float().cpu(), torch.ones(H, dtype=torch.bool)
            for c, number in zip(columns, (math.inf, -math.inf, math.nan)):
                at = range(c // 32 * 32, min(H, c // 32 * 32 + 32)) if math.isnan(number) and fmt != "bf16" else [c]
                for i in at:
                    rest[i] = False
                    y = got[..., i][sees]
                    assert bool((torch.isnan(y) if math.isnan(number) else y == number).all()), (fmt, normalised, call.__name__, i, number)
            want = sees.unsqueeze(-1) & ~rest
            assert torch.equal(torch.where(want, 0.0, got), torch.where(want, 0.0, before[0].float().cpu()))
