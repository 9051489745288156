"""How calls under score rules go out (binding.scored_route: the library's own plans, on the CPU), and that the GPU tests' cases take the
forms that they are there for.  256 compute units, as on MI355X."""
import random

import pytest

from test_gpu_scored_forms import BACKWARD, FINE, FORWARD, name_of

CUS = 256


@pytest.fixture(scope="module")
def a2d():
    from paper_2503_15758_amd import binding
    binding._ext()
    return binding


def route(a2d, heads, kvh, nq, nkv, H, more, **kw):
    rules = {k: more[k] for k in ("q_off", "kv_off", "causal", "softcap") if k in more}
    return a2d.scored_route(heads, nq, nkv, H, kv_heads=kvh, slopes="slopes" in more,
                            range_sets=len(more["lens"]) if "lens" in more else int("docs" in more), compute_units=CUS, **rules, **kw)


@pytest.mark.parametrize("case", FORWARD, ids=name_of)
def test_forward_forms(a2d, case):
    form, order, split = case[6:]
    r = route(a2d, *case[:6])
    assert (r["rows"], r["lanes"], r["waves"]) == form and r["order"] == order
    assert (r["units_q"] > r["blocks_q"]) == split and r["kernels"] == ("scored_fwd_kernel",) + ("fix_kernel",) * split


@pytest.mark.parametrize("case", BACKWARD, ids=name_of)
def test_backward_forms(a2d, case):
    lanes, shared_q, cut_q, shared_kv, cut_kv = case[6:]
    r = route(a2d, *case[:6], backward=True)
    assert (r["lanes"], r["rows"]) == (lanes, 256 // lanes)
    assert (r["shared_q"], r["units_q"] > r["blocks_q"]) == (shared_q, cut_q)
    assert (r["shared_kv"], r["units_kv"] > r["blocks_kv"]) == (shared_kv, cut_kv)
    assert ("scored_sum_kernel" in r["kernels"]) == (cut_q or cut_kv)


def test_every_form_is_there():
    forms = {c[6] for c in FORWARD}
    assert len(forms) == 3 and len({(c[6], c[8]) for c in FORWARD}) == 6
    assert len({(c[6], c[4]) for c in FORWARD}) == 12                              # head sizes
    for rule in ("slopes", "softcap"):
        assert len({(c[6], rule in c[5]) for c in FORWARD}) == 6


def test_without_memory_nothing_is_in_parts(a2d):
    rng = random.Random(2)
    for _ in range(300):
        kv = int(2 ** rng.uniform(0, 5))
        heads = kv * rng.choice([1, 1, 4])
        nq, nkv = (int(2 ** rng.uniform(0, 13)) for _ in range(2))
        more = dict(causal=rng.random() < 0.5, **(dict(docs=()) if rng.random() < 0.4 else {}))
        for backward in (False, True):
            r = route(a2d, heads, kv, nq, nkv, 128, more, backward=backward, scratch=False)
            assert r["units_q"] == r["blocks_q"] and r["units_kv"] == r["blocks_kv"], (heads, kv, nq, nkv, more)


@pytest.mark.parametrize("case", FINE, ids=name_of)
def test_two_numbers(a2d, case):
    for scratch in (False, True):
        r = route(a2d, *case, scratch=scratch)
        assert r["fine"] and r["kernels"][0] == "scored_fwd_small_kernel"


def test_rounding_does_not_go_by_memory(a2d):
    """The results of a call without memory for partial results are the same up to the order of fp32 sums: P and dZ are rounded alike.  Up to 32
    rows for each key/value head are taken as two numbers, in a forward, and up to 2^22 scores in a backward."""
    rng, kinds = random.Random(3), set()
    for _ in range(3000):
        kv = int(2 ** rng.uniform(0, 6))
        heads = kv * rng.choice([1, 1, 2, 4, 8])
        nq, nkv = int(2 ** rng.uniform(0, rng.choice([5, 13]))), int(2 ** rng.uniform(4, 14))
        more = dict(causal=rng.random() < 0.4, q_off=rng.randint(0, nkv), **(dict(slopes=True) if rng.random() < 0.5 else {}),
                    **rng.choice([dict(), dict(docs=()), dict(lens=[1] * kv)]))
        case = (heads, kv, nq, nkv, rng.choice([64, 80, 96, 128]), more)
        with_, without = (route(a2d, *case, scratch=x) for x in (True, False))
        assert with_["fine"] == without["fine"], case
        assert with_["fine"] == (with_["kernels"][0] == "scored_fwd_small_kernel"), case
        if (heads // kv if heads > kv else 1) * nq <= 32:
            assert with_["fine"], case
        kinds.add((with_["fine"], with_["kernels"][0] == without["kernels"][0], without["kernels"][0]))
        if nkv > 1:
            assert route(a2d, *case, backward=True)["fine"] == (heads * nq * nkv <= 1 << 22)
    assert len(kinds) == 3, kinds                                                   # (other forms without memory among them)


def test_one_sequence_is_no_documents(a2d):
    """A set of ranges for a few new rows is a cache's filled length as well: they are planned for all of it, as without ranges, or in a batch
    with another sequence."""
    rng = random.Random(4)
    same = ("kernels", "rows", "lanes", "waves", "blocks_q", "units_q", "blocks_kv", "units_kv", "shared_q", "shared_kv")
    for _ in range(500):
        kv = 2 * int(2 ** rng.uniform(0, 5))
        case = (kv * rng.choice([1, 1, 4]), kv, int(2 ** rng.uniform(0, 7)), int(2 ** rng.uniform(4, 14)), rng.choice([64, 80, 96, 128]))
        for backward in (False, True):
            one, none, two = (route(a2d, *case, dict(lens=[case[3]] * n) if n else {}, backward=backward) for n in (1, 0, 2))
            for k in same:
                assert one[k] == none[k] == two[k], (case, backward, k)
