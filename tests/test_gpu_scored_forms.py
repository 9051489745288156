"""The bf16 calls under score rules in every form of their kernels, each at a size that the library's plans send there
(test_host_scored_routes.py holds them to it, on the CPU): forwards of 256 rows, of 128 in two key lanes and in workgroups of four
wavefronts, with walks whole and in parts; gradients whose row blocks are shared out in proportion to their walks.  Bounds:
tests/scored_reference.py."""
import pytest
import torch

import scored_reference
from scored_reference import Scored, half_step, within
from test_gpu_scored import check_fwd, documents, inputs, int32, slopes_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# rows, key lanes and wavefronts of a workgroup
BIG, LANES, PAIRS = (256, 1, 8), (128, 2, 8), (128, 1, 4)
HEADS, LATE, RANKED = 0, 1, 2                          # order of the blocks
STEEP = [8.0, 0.5, -0.01, 1e-6, 30.0, -0.25, 0.0, 3.0]  # slopes of eight heads
DOCS = ([0, 300, 730, 760, 1010, 1290], [20, 0, 500, 7, 0])

# heads, kv_heads, nq, nkv, H, rules | form, order, walks in parts
FORWARD = [
    (24, 3, 1300, 65, 64, dict(slopes=True), BIG, HEADS, False),
    (24, 3, 1300, 65, 80, dict(softcap=4.0, slopes=True), BIG, HEADS, False),
    (24, 3, 1300, 65, 96, dict(), BIG, HEADS, False),
    (32, 8, 1025, 65, 128, dict(softcap=9.0, slopes=True, causal=True), BIG, LATE, False),
    (40, 8, 1300, 65, 64, dict(docs=DOCS, kv_off=715, slopes=True), BIG, RANKED, False),
    (40, 8, 1300, 65, 96, dict(docs=DOCS, kv_off=740, softcap=9.0), BIG, RANKED, False),
    (64, 8, 129, 1000, 80, dict(softcap=20.0), BIG, HEADS, True),
    (64, 8, 129, 800, 64, dict(softcap=20.0, slopes=True, q_off=600), BIG, HEADS, True),
    (64, 8, 129, 1300, 128, dict(slopes=STEEP * 8, q_off=500), BIG, HEADS, True),
    (16, 4, 1025, 450, 128, dict(softcap=20.0), LANES, HEADS, False),
    (40, 8, 400, 600, 64, dict(softcap=5.0, slopes=True, q_off=100), LANES, HEADS, False),
    (40, 8, 400, 450, 96, dict(slopes=STEEP * 5, softcap=20.0, q_off=30), LANES, HEADS, False),
    (4, 4, 4100, 450, 128, dict(slopes=STEEP[:4], q_off=-2000), LANES, HEADS, False),
    (5, 5, 4100, 450, 96, dict(softcap=20.0, slopes=True, causal=True), LANES, LATE, False),
    (40, 8, 200, 1300, 128, dict(softcap=20.0), LANES, HEADS, True),
    (40, 8, 200, 1300, 96, dict(softcap=20.0, slopes=STEEP * 5, q_off=700), LANES, HEADS, True),
    (1, 1, 4100, 3000, 80, dict(softcap=7.0, slopes=True), LANES, HEADS, True),
    (1, 1, 4100, 3000, 64, dict(softcap=7.0, slopes=STEEP[4:5]), LANES, HEADS, True),
    (40, 8, 200, 700, 64, dict(slopes=STEEP * 5, q_off=300), PAIRS, HEADS, True),
    (40, 8, 200, 65, 64, dict(slopes=STEEP * 5), PAIRS, HEADS, False),
    (4, 4, 1025, 65, 64, dict(slopes=True, causal=True), PAIRS, LATE, False),
    (1, 1, 129, 1300, 96, dict(softcap=20.0), PAIRS, HEADS, True),
    (1, 1, 129, 1300, 80, dict(), PAIRS, HEADS, True),
    (2, 1, 130, 4000, 64, dict(docs=([0, 1900, 2000, 2060, 4000], [0, 70, 5, 9]), softcap=20.0, slopes=True, q_off=1940), PAIRS, RANKED, True),
    (1, 1, 129, 4000, 128, dict(docs=([0, 3900, 4000], [1, 0]), softcap=20.0, q_off=3830), PAIRS, RANKED, True),
]


def name_of(c):
    return "_".join(["%dx%dx%dx%d_H%d" % c[:5]] + sorted(c[5]))


def rules_of(a2d, heads, nq, more):
    rules = {k: v for k, v in more.items() if k != "docs"}
    if "slopes" in rules:
        rules["slopes"] = slopes_of(heads) if rules["slopes"] is True else torch.tensor(rules["slopes"], device="cuda")
    if "docs" in more:
        rules["ranges"] = documents(a2d, nq, *more["docs"], first=rules.get("q_off", 0))
    return rules


@pytest.fixture(scope="module")
def a2d():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_15758_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("case", FORWARD, ids=name_of)
def test_forward(a2d, case):
    heads, kvh, nq, nkv, H, more = case[:6]
    print("scored forward form", case, flush=True)
    Q, K, V, _ = inputs(heads, kvh, nq, nkv, H, "bf16")
    rules = rules_of(a2d, heads, nq, more)
    ref = Scored(Q, K, V, **rules).partial()
    for norm in (False, True):
        got = a2d.partial_fwd_scored(Q, K, V, normalised=norm, **rules)
        check_fwd(got, ref, norm, Q.dtype, str(case[:6]))
        assert all(torch.equal(x, y) for x, y in zip(got, a2d.partial_fwd_scored(Q, K, V, normalised=norm, **rules))), "not reproducible"


@pytest.mark.parametrize("case", FORWARD, ids=name_of)
def test_forward_accumulated(a2d, case):
    """The call continues the partial of the keys behind its own: of 70 more, which the form depends on as little as they add time."""
    heads, kvh, nq, nkv, H, more = case[:6]
    print("scored forward form, accumulated", case, flush=True)
    Q, K, V, _ = inputs(heads, kvh, nq, nkv + 70, H, "bf16")
    rules = rules_of(a2d, heads, nq, more)
    off = rules.pop("kv_off", 0)
    out = a2d.partial_fwd_scored(Q, K[:, nkv:], V[:, nkv:], kv_off=off + nkv, **rules)
    a2d.partial_fwd_scored(Q, K[:, :nkv], V[:, :nkv], kv_off=off, out=out, accumulate=True, **rules)
    ref = Scored(Q, K, V, kv_off=off, **rules).partial()
    # (two calls: each rounding once in either, the stored partial's reference once more)
    check_fwd(out, {k: v * 2 if k.startswith("e_") else v for k, v in ref.items()}, False, Q.dtype, str(case[:6]))


# heads, kv_heads, nq, nkv, H, rules | key lanes of dQ, its blocks shared out, cut; those of dK / dV shared out, cut
BACKWARD = [
    (1, 1, 3200, 3000, 128, dict(docs=([0, 40, 1100, 1111, 3100], [0, 900, 3, 64]), softcap=20.0, slopes=True), 2, True, True, True, True),
    (4, 4, 2100, 1500, 128, dict(docs=([0, 700, 701, 2000], [500, 1, 0]), softcap=20.0, slopes=True), 2, True, True, True, True),
    (5, 5, 4100, 1000, 128, dict(docs=([0, 100, 900, 4000], [0, 800, 0])), 2, True, False, True, True),
    (5, 5, 4100, 1000, 96, dict(docs=([0, 100, 900, 4000], [0, 800, 0])), 1, True, True, True, True),
    (8, 8, 513, 1500, 128, dict(docs=([0, 1000, 1200, 1500], [0, 9, 30]), q_off=980), 2, False, True, True, False),
    (6, 3, 130, 65, 64, dict(), 1, False, False, False, True),
    (8, 8, 130, 450, 128, dict(), 1, False, True, False, False),
]


@pytest.mark.parametrize("case", BACKWARD, ids=name_of)
def test_backward(a2d, case):
    heads, kvh, nq, nkv, H, more = case[:6]
    print("scored backward form", case, flush=True)
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, "bf16")
    rules = rules_of(a2d, heads, nq, more)
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    want = s.gradients(O, dO, lse)
    del s, f
    for rounded in (False, True):
        got = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=rounded, **rules)
        for x, n in zip(got, ("dQ", "dK", "dV")):
            within(x, want[n], want["e_" + n], "%s %s" % (case[:6], n), half_step(Q.dtype) if rounded else 0.0)
        again = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, rounded=rounded, **rules)
        assert all(torch.equal(x, y) for x, y in zip(got, again)), "not reproducible"
    plain = a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules)
    out = tuple(torch.full_like(x, 1.0, dtype=torch.float32) for x in (Q, K, V))
    a2d.partial_bwd_scored(Q, K, V, O, dO, lse, out=out, accumulate=True, **rules)
    # (1 is added first, or last: each of up to 33 partial sums is rounded next to it)
    within(out[0], plain[0].cpu().double() + 1.0, 40 * U * (1.0 + plain[0].cpu().double().abs()), "accumulated")
    assert torch.equal(out[1], plain[1]) and torch.equal(out[2], plain[2])


# ---- P and dZ as two bf16 numbers each: h = x rounded to bf16, x - h is exact and below 2^-8 of x's power of two, so rounded it is off by
# 2^-17 of x.  The sums' other errors as ever.
TWO = 2.0 ** -17

# heads, kv_heads, nq, nkv, H, rules ("lens": the lengths of caches, one for each run of heads)
FINE = [
    (32, 8, 1, 1133, 128, dict(softcap=30.0, lens=[1133])),
    (32, 8, 1, 1133, 128, dict(softcap=30.0)),
    (8, 2, 1, 2048, 128, dict(lens=[2048])),
    (8, 8, 1, 4096, 96, dict(lens=[4001], slopes=True, q_off=4000)),
    (12, 12, 5, 1300, 64, dict(lens=[1300, 40, 777])),
    (2, 2, 1, 104, 64, dict(lens=[104])),
    (16, 4, 8, 900, 80, dict(causal=True, q_off=892, softcap=8.0, slopes=True)),
    (1, 1, 32, 5000, 128, dict(slopes=STEEP[4:5], q_off=4968)),
    (2, 1, 130, 1000, 80, dict(softcap=20.0)),
]


def fine_rules(heads, nq, more):
    rules = rules_of(None, heads, nq, {k: v for k, v in more.items() if k != "lens"})
    if "lens" in more:
        rules["ranges"] = int32([[[0, n]] * nq for n in more["lens"]])
    return rules


@pytest.mark.parametrize("case", FINE, ids=name_of)
def test_probabilities_as_two_numbers(a2d, monkeypatch, case):
    heads, kvh, nq, nkv, H, more = case
    print("two numbers", case, flush=True)
    Q, K, V, _ = inputs(heads, kvh, nq, nkv, H, "bf16", sigma=3.0 if "softcap" in more else 1.0)
    rules = fine_rules(heads, nq, more)
    s = Scored(Q, K, V, **rules)
    with monkeypatch.context() as m:
        m.setattr(scored_reference, "half_step", lambda dtype: TWO)
        ref = s.partial()
    # (one number would be outside; a row whose weight one key has holds 1, which is one)
    w = torch.exp(s.s - ref["m"].unsqueeze(2))
    once = w.bfloat16().double() @ s.V / ref["l"].unsqueeze(2)
    assert ((once - ref["O"]).abs() > ref["e_O"]).any() or ref["l"].max() < 1 + 2.0 ** -20
    check_fwd(a2d.partial_fwd_scored(Q, K, V, **rules), ref, False, Q.dtype, str(case))
    out = (torch.zeros(heads, nq, H, device="cuda"), torch.full((heads, nq), -float("inf"), device="cuda"), torch.zeros(heads, nq, device="cuda"))
    check_fwd(a2d.partial_fwd_scored(Q, K, V, out=out, accumulate=True, **rules), ref, False, Q.dtype, str(case))


@pytest.mark.parametrize("case", [(32, 8, 40, 100, 128, dict(softcap=30.0)), (4, 1, 349, 193, 80, dict(slopes=True, q_off=20)), (2, 2, 1000, 700, 64, dict(causal=True)),
                                  (3, 3, 300, 290, 96, dict(docs=DOCS, softcap=9.0, slopes=True))], ids=name_of)
def test_gradients_as_two_numbers(a2d, monkeypatch, case):
    heads, kvh, nq, nkv, H, more = case
    print("two numbers, gradients", case, flush=True)
    Q, K, V, dO = inputs(heads, kvh, nq, nkv, H, "bf16")
    rules = rules_of(a2d, heads, nq, more)
    s = Scored(Q, K, V, **rules)
    f = s.partial()
    O, lse = f["O"].to(Q.dtype).cuda(), f["lse"].float().cuda()
    with monkeypatch.context() as m:
        m.setattr(scored_reference, "half_step", lambda dtype: TWO)
        want = s.gradients(O, dO, lse)
    g, L = dO.cpu().double(), lse.cpu().double().unsqueeze(2)
    p = torch.exp(s.s - L).nan_to_num(0.0)
    dz = s.scale * p * (g @ s.V.transpose(1, 2) - (g * O.cpu().double()).sum(2, keepdim=True)) * s.dy
    by_kv = lambda x: x.view(-1, s.group, *x.shape[1:]).sum(1)
    for n, once in (("dQ", dz.bfloat16().double() @ s.K), ("dK", by_kv(dz.bfloat16().double().transpose(1, 2) @ s.Q)),
                    ("dV", by_kv(p.bfloat16().double().transpose(1, 2) @ g))):
        assert ((once - want[n]).abs() > want["e_" + n]).any(), n
    for x, n in zip(a2d.partial_bwd_scored(Q, K, V, O, dO, lse, **rules), ("dQ", "dK", "dV")):
        within(x, want[n], want["e_" + n], "%s %s" % (case, n))
