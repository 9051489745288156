"""Scores of any size that fp32 holds: scales up to the largest that is accepted, large Q and K, scores near the lowest number."""
import math

import pytest
import torch

import cached_reference as ref
from cached_calls import without_workspace
from test_gpu_cached_attention import _call, _problem, kernels  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

FORMS = [(1, 1), (4, 5), (2, 40), (2, 80)]


def _whole(seed, fmt, H, group, rows, lens, power=0):
    """Q, K and V of whole numbers from -2 to 2 (Q and K times 2^power), which every format holds and whose scores fp32 sums exactly."""
    x = _problem(seed, fmt, H, 1, group, rows, lens, 16, masked=rows > 1)
    gen = torch.Generator().manual_seed(seed + 100)
    draw = lambda shape: torch.randint(-2, 3, shape, generator=gen).float()
    for name in ("Q", "K", "V"):
        x[name] = (draw(x[name].shape) * (1.0 if name == "V" else 2.0 ** power)).bfloat16().cuda()
    shape = (*x["cache"][0].shape[:3], H)
    cache, scales = [], []
    for i in range(2):
        y = draw(shape) * (1.0 if i else 2.0 ** power)
        if fmt == "bf16":
            cache.append(y.bfloat16().cuda())
            continue
        codes, e = ref.quantised(y, fmt)
        c = codes.to(torch.uint8).view(torch.float8_e4m3fn) if fmt == "e4m3" else (codes[..., 0::2] + 16 * codes[..., 1::2]).to(torch.uint8)
        s = torch.full((*e.shape[:-1], 4), 127, dtype=torch.uint8)
        s[..., :e.shape[-1]] = (e + 127).to(torch.uint8)
        cache.append(c.cuda())
        scales.append(s.cuda())
    x["cache"] = tuple(cache + scales)
    assert all(torch.equal(ref.cache_values(x["cache"], i), ref.cache_values(x["cache"], i).round()) for i in range(2)) or power < 0
    return x


def _exactly(x):
    """The definition in 64 bits.  Scores differ by the scale's size or not at all, so a row is the mean of its largest keys' V: sums of equal
    probabilities.  m: the scale, log2 e, their product, the score's product with it, ln 2 and the product with that, each rounded by 2^-24 at the
    most: 2^-21 of it.  N and l are relative to such a number of log2 units, whose half step is 2^-24 of it: a factor of 2^h, h that half step, as long as
    exponents are taken from the unrounded product; never more than 2 (half a step of at most 1), and 1 where the products are rounded alike.
    O: that factor cancels, P as one bf16 number 2^-8 at the most, the result half a step, sums of up to 2^12 terms 2^-12."""
    N, m, l, A, size = ref.attention(x["Q"], [ref.cache_values(x["cache"], i) for i in range(2)], x["table"], x["lens"], x["K"], x["V"], x["masks"],
                                     x["scale"])
    some = l > 0
    one = torch.where(some, l, torch.ones_like(l))
    O = N / one.unsqueeze(-1)
    top = torch.where(some, m, torch.zeros_like(m))
    factor = torch.exp2((top.abs() * 1.4427 * 2.0 ** -24).clamp(max=1.0)) * (1 + 2.0 ** -15)
    for call in (_call, without_workspace):
        o, lse = (y.double().cpu() for y in call(x, normalised=True))
        assert bool(((o - O).abs() <= (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -12) * (A / one.unsqueeze(-1))).all()), call.__name__
        assert torch.equal(lse == -math.inf, ~some)
        # (beside a large m, log l is part of its rounding)
        assert bool(((lse - top - torch.log(one)).abs() <= 2.0 ** -20 * top.abs() + 2.0 ** -14)[some].all())
        n2, m2, l2 = (y.double().cpu() for y in call(x))
        assert torch.equal(m2 == -math.inf, ~some) and bool((l2[~some] == 0).all())
        assert bool(((m2 - top).abs() <= 2.0 ** -21 * top.abs())[some].all())
        assert bool(((l2 <= l * factor) & (l2 * factor >= l))[some].all()), call.__name__
        # (N and l have the same factor)
        f = torch.where(some, l2 / one, torch.ones_like(l)).unsqueeze(-1)
        assert bool(((n2 - N * f).abs() <= 2.0 ** -12 * A * f).all())


@pytest.mark.parametrize("scale", [1e4, 1e5, 1e6, 1e7, 1e9, 1e12, 1e20, 1e30])
@pytest.mark.parametrize("group, rows", FORMS)
def test_large_scales(kernels, scale, group, rows):
    x = _whole(1, "e4m3", 64, group, rows, [1200, 70, 0, 33])
    x["scale"] = scale
    _exactly(x)


@pytest.mark.parametrize("fmt, H", [("bf16", 128), ("e4m3", 80), ("e2m1", 96)])
@pytest.mark.parametrize("power", [10, 20, 45])
@pytest.mark.parametrize("group, rows", FORMS)
def test_large_keys(kernels, fmt, H, power, group, rows):
    x = _whole(2, fmt, H, group, rows, [900, 5], power)
    x["scale"] = 1 / math.sqrt(H)
    _exactly(x)


@pytest.mark.parametrize("scale", [1e3, 1e6, 1e8, 1e9, 1e10, 1e12, 1e18, 1e30])
@pytest.mark.parametrize("group, rows", FORMS)
def test_rows_stay_rows(kernels, scale, group, rows):
    """Scores that are rounded: which key is the largest may be another one, but a row's largest probability is 1, or within 2 of it, and O lies
    between the smallest and the largest V (half a step of the result and of P each 2^-8)."""
    x = _problem(3, "e4m3", 96, 1, group, rows, [1500, 40], 48, masked=False, sigma=3.0)
    x["scale"] = scale
    most = max(float(ref.cache_values(x["cache"], 1).abs().max()), float(x["V"].float().abs().max()))
    for call in (_call, without_workspace):
        O, lse = call(x, normalised=True)
        assert bool(torch.isfinite(lse).all()) and bool((O.float().abs() <= most * (1 + 2.0 ** -6)).all())
        N, m, l = call(x)
        assert bool((l >= 0.5).all()) and bool((l <= 2 * (1500 + rows)).all()) and bool(torch.isfinite(m).all())
        assert bool((N.abs() <= l.unsqueeze(-1) * most * (1 + 2.0 ** -12)).all())


@pytest.mark.parametrize("group, rows", FORMS)
@pytest.mark.parametrize("size", [2.0, -2.0, 0.8125, -0.8125])
def test_next_to_the_ends_of_fp32(kernels, group, rows, size):
    """One key, whose score in log2 units is near 2^128, up and down: it is all that the row has."""
    x = _problem(4, "bf16", 64, 1, group, rows, [1, 0], 16, masked=False, drafts=False)
    x["cache"][0].zero_()
    x["cache"][0][..., 5] = size * 2.0 ** 13
    x["Q"] = torch.zeros_like(x["Q"])
    x["Q"][..., 5] = 2.0 ** (14 if abs(size) > 1 else 15)
    x["scale"] = 0.8125e30 if abs(size) > 1 else 1e30       # log2 units: 3.14e38 of 3.40e38
    want = ref.cache_values(x["cache"], 1)[int(x["table"][0, 0]), 0, 0]
    score = size * 2.0 ** 13 * float(x["Q"][0, 0, 0, 5]) * x["scale"]
    assert 3.0e38 < abs(score) * math.log2(math.e) < 3.4e38
    for call in (_call, without_workspace):
        N, m, l = (y.double().cpu() for y in call(x))
        assert bool((l[0] == 1).all()) and bool((N[0] == want).all()) and bool(((m[0] - score).abs() <= 2.0 ** -21 * abs(score)).all())
        assert bool((l[1] == 0).all()) and bool((m[1] == -math.inf).all())
        O, lse = call(x, normalised=True)
        assert bool((O[0].double().cpu() == want).all())
