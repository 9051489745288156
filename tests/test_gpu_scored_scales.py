"""Capped scores of inputs far from 1 in size, which a scale far from 1 / sqrt(H) brings back: the powers of scale / softcap, and of the raw
products, that the cap's polynomial is made of leave fp32's range.  Bounds: tests/scored_reference.py."""
import pytest
import torch

from scored_reference import Scored, half_step, within
from test_gpu_scored import check_fwd, inputs, slopes_of

pytestmark = pytest.mark.gpu

# scale, cap, size of Q, of K: scores of a third to a half of the cap, and beyond
SIZES = [(1e-8, 30.0, 1e4, 1e4), (1e-13, 2.0, 1e6, 1e6), (2e-20, 1.0, 2e9, 1e9), (1e-6, 1e-4, 0.1, 30.0), (40.0, 3.0, 0.03, 0.1), (1e-5, 50.0, 2e3, 200.0)]
# heads, kv_heads, nq, nkv, H, type
SHAPES = [(4, 2, 300, 470, 64, "bf16"), (24, 3, 1300, 65, 96, "bf16"), (16, 4, 1025, 450, 128, "bf16"), (8, 2, 1, 500, 128, "bf16"),
          (4, 2, 150, 203, 96, "f32"), (6, 6, 1, 300, 64, "f32")]


@pytest.fixture(scope="module", params=["default", "generic"])
def a2d(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding
    binding.lib()
    binding.force_generic(request.param == "generic")
    yield binding
    binding.force_generic(False)


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "scale%g_cap%g" % s[:2])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%dx%dx%d_H%d_%s" % s)
def test_scales(a2d, shape, sizes):
    heads, kvh, nq, nkv, H, dt = shape
    scale, cap, of_q, of_k = sizes
    print("scored scales", shape, sizes, flush=True)
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, dt)
    Q, K = Q * of_q, K * of_k
    for rules in (dict(softcap=cap, scale=scale), dict(softcap=cap, scale=scale, slopes=slopes_of(heads), q_off=50, causal=True)):
        s = Scored(Q, K, V, **rules)
        f = s.partial()
        check_fwd(a2d.partial_fwd_scored(Q, K, V, normalised=True, **rules), f, True, Q.dtype, "scale")
        if nq == 1:
            continue
        O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
        want = s.gradients(O, dO, lse)
        for x, n in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules), ("dQ", "dK", "dV")):
            within(x, want[n], want["e_" + n], "scale %s" % n)


@pytest.mark.parametrize("step, slope, nq, nkv", [(4, 0.7, 300, 187), (1, 8.0, 200, 90), (1000, 0.01, 77, 300), (1, 0.0, 150, 203)])
def test_fp32_gradients_far_from_the_keys(a2d, step, slope, nq, nkv):
    """Rows thousands of units of bias behind their keys: bias and lse cancel, and P is off by the roundings of what is left.  Scores of nothing but
    the bias, so that P = exp(-slope d - lse) is known from fp32 numbers: dV = P^T dO.  Each P is off by 2^-24 of |slope d + lse|
    twice (that sum's rounding, and log2(e) times it) and some 8 half steps, the sum over rows by (nq + 16) more."""
    H, u = 64, 2.0 ** -24
    gen = torch.Generator().manual_seed(4)
    K, V, dO = (torch.randn(2, n, H, generator=gen).cuda() for n in (nkv, nkv, nq))
    Q, slopes, off = torch.zeros(2, nq, H, device="cuda"), torch.tensor([slope, slope / 3], device="cuda"), 700 * step
    s = Scored(Q, K, V, slopes=slopes, q_off=off, token_step=step)
    lse = s.partial()["lse"].float().cuda()
    rest = s.s - lse.cpu().double().unsqueeze(2)
    p = torch.exp(rest)
    _, _, dV = a2d.partial_bwd_scored(Q, K, V, torch.zeros_like(Q), dO, lse, slopes=slopes, q_off=off, token_step=step)
    g = dO.cpu().double()
    bound = (p * ((nq + 24) * u + 4 * u * rest.abs())).transpose(1, 2) @ g.abs()
    within(dV, p.transpose(1, 2) @ g, bound, "dV")
