"""Sines and cosines of rotary positions by themselves - (1, 0) turned - against rational arithmetic: relative to their own size, next to whole
and half turns too.  Bounds: sine_cosine in a2d_rotary.hip says 4 half steps of fp32 (the angle's rounding, 2 pi's, the product's, the
last sum's), 2^-64 turns a position of the frequency, and the result's own rounding."""
import math
from fractions import Fraction

import pytest
import torch

from scored_reference import half_step
from test_gpu_scored import int32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def arctan(x):                                       # of 1 / x, in units of 2^-300
    total = term = (1 << 300) // x
    n, sign = 3, -1
    while term:
        term //= x * x
        total += sign * (term // n)
        n, sign = n + 2, -sign
    return total


TURN = Fraction(8 * (4 * arctan(5) - arctan(239)), 1 << 300)


def exact(position, freq):
    """(cos, sin), each good to 2^-50 of itself: from the nearest quarter turn."""
    part = (position * Fraction(freq) / TURN) % 1
    quarter = round(part * 4)
    rest = 2 * math.pi * float(part - Fraction(quarter, 4))
    c, s = math.cos(rest), math.sin(rest)
    return [(c, s), (-s, c), (-c, -s), (s, -c)][quarter % 4]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_sines_and_cosines(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding as a2d
    H = 128
    freqs = [10000.0 ** (-2.0 * p / H) for p in range(60)] + [math.pi, -math.pi / 2, 2 * math.pi, 1e-12]
    rows = [0, 1, 2, 3, 7, 22, -1, 100, 355, 710, 4096, 103993, -104348, 1 << 20, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31]
    X = torch.zeros(1, len(rows), H, dtype=dtype, device="cuda")
    X[:, :, :64] = 1.0
    got = a2d.rotary(X, int32([rows]), torch.tensor(freqs, dtype=torch.float64)).cpu().double()[0]
    r = half_step(dtype) or U
    for i, n in enumerate(rows):
        for p, f in enumerate(freqs):
            for x, want in zip((got[i, p].item(), got[i, 64 + p].item()), exact(n, f)):
                bound = (4 * U + r + 4 * U * r) * abs(want) + 2 * math.pi * abs(n) * 2.0 ** -64 * (1 + r)
                assert abs(x - want) <= bound, (n, f, x, want)
