"""What the calls under score rules and the rotary call refuse, on the CPU: with bad arguments nothing is enqueued."""
import ctypes
import os
import subprocess

import pytest
import torch

P = ctypes.c_void_p(0x10000)                       # aligned, never dereferenced: every call here fails its checks
ODD = ctypes.c_void_p(0x10008)
NULL = None
INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module")
def b():
    from paper_2503_15758_amd import binding
    binding.lib()
    return binding


def desc(b, **kw):
    d = dict(heads=4, nq=128, nkv=128, hdim=128, q_off=0, kv_off=0, causal=0, scale=0.1, dtype=b.A2D_BF16)
    d.update(kw)
    return b.TileDesc(**d)


def rules(b, **kw):
    r = dict(softcap=30.0, token_step=1, range_sets=1, pad=0, slopes=P, ranges=P)
    r.update(kw)
    return b.ScoreRules(**r)


def fwd(b, d=None, r=None, kvh=2, flags=0, q=P, out=(P, P, P)):
    return b.lib().a2d_partial_fwd_scored(d and ctypes.byref(d), kvh, r and ctypes.byref(r), flags, q, P, P, *out, NULL, 0, NULL)


def bwd(b, d, r, kvh=2, flags=0, lse=P, ws=P, wb=1 << 20):
    return b.lib().a2d_partial_bwd_scored(ctypes.byref(d), kvh, ctypes.byref(r), flags, P, P, P, P, P, lse, P, P, P, ws, wb, NULL)


BAD_RULES = [(dict(softcap=-1.0), INVALID), (dict(softcap=float("nan")), INVALID), (dict(softcap=float("inf")), INVALID),
             (dict(softcap=1e-9), UNSUPPORTED), (dict(softcap=1e9), UNSUPPORTED), (dict(token_step=0), INVALID),
             (dict(token_step=(1 << 20) + 1), INVALID), (dict(pad=1), INVALID), (dict(range_sets=0), INVALID),
             (dict(range_sets=3), INVALID), (dict(range_sets=4), INVALID), (dict(slopes=ODD), MISALIGNED), (dict(ranges=ODD), MISALIGNED)]


@pytest.mark.parametrize("change, status", BAD_RULES, ids=lambda x: str(x))
def test_bad_rules(b, change, status):
    assert fwd(b, desc(b), rules(b, **change)) == status
    assert bwd(b, desc(b), rules(b, **change)) == status
    assert b.lib().a2d_last_error()


def test_bad_tiles_and_pointers(b):
    r = rules(b)
    assert fwd(b, None, r) == INVALID and fwd(b, desc(b), None) == INVALID
    for kvh in (0, 3, -1, 8):
        assert fwd(b, desc(b), r, kvh=kvh) == INVALID
    for change, status in ((dict(nq=0), INVALID), (dict(nkv=0), INVALID), (dict(hdim=72), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
                           (dict(scale=0.0), INVALID), (dict(causal=2), INVALID), (dict(scale=1e30), UNSUPPORTED)):
        assert fwd(b, desc(b, **change), r) == status, change
    for flags in (3, 4, 8, -1):
        assert fwd(b, desc(b), r, flags=flags) == INVALID and bwd(b, desc(b), r, flags=flags) == INVALID
    assert fwd(b, desc(b), r, q=NULL) == INVALID and fwd(b, desc(b), r, q=ODD) == MISALIGNED
    assert fwd(b, desc(b), r, out=(P, P, NULL)) == INVALID
    assert bwd(b, desc(b), r, lse=NULL) == INVALID
    assert bwd(b, desc(b, flags=b.DESC_KEEP_DS), r) == UNSUPPORTED


def test_scales_too_small(b):
    """lse / scale is formed in fp32"""
    assert fwd(b, desc(b, scale=9e-21), rules(b)) == UNSUPPORTED and bwd(b, desc(b, scale=1e-38), rules(b, softcap=0.0)) == UNSUPPORTED
    assert fwd(b, desc(b, scale=1.1e-20), rules(b, softcap=0.0), q=ODD) == MISALIGNED


def test_distances_of_a_bias(b):
    """Up to 2^24 tokens: they are fp32 in the kernels."""
    for change in (dict(q_off=(1 << 24) - 126), dict(kv_off=(1 << 24) - 126)):
        assert fwd(b, desc(b, **change), rules(b)) == UNSUPPORTED
    assert fwd(b, desc(b, q_off=1 << 30), rules(b, token_step=1 << 20)) == UNSUPPORTED
    # (the checks behind it are reached where the distances fit, or where there is no bias)
    assert fwd(b, desc(b, q_off=(1 << 24) - 127), rules(b), q=ODD) == MISALIGNED
    assert fwd(b, desc(b, q_off=1 << 39), rules(b, slopes=NULL), q=ODD) == MISALIGNED


def test_workspace(b):
    d = desc(b)
    need = b.workspace_bytes(d, b.OP_PARTIAL_BWD_SCORED)
    assert need == 4 * 128 * 16 + 4 * 4 * 32       # 16 bytes a row, 32 for each 32 rows; rows up to a multiple of 64
    assert b.workspace_bytes(desc(b, heads=3, nq=65), b.OP_PARTIAL_BWD_SCORED) == b.workspace_bytes(desc(b, heads=3), b.OP_PARTIAL_BWD_SCORED)
    assert bwd(b, d, rules(b), wb=need - 1) == WORKSPACE and bwd(b, d, rules(b), ws=NULL) == WORKSPACE
    assert bwd(b, d, rules(b), ws=ODD) == MISALIGNED and bwd(b, d, rules(b), wb=1 << 60) == INVALID


def test_document_ranges(b):
    f = b.lib().a2d_document_ranges
    good = dict(documents=3, starts=P, prefix=NULL, causal=1, first=0, step=1, rows=10, ranges=P)
    for change, status in ((dict(documents=0), INVALID), (dict(rows=0), INVALID), (dict(rows=(1 << 22) + 1), INVALID), (dict(step=0), INVALID),
                           (dict(causal=2), INVALID), (dict(first=1 << 50), INVALID), (dict(starts=NULL), INVALID),
                           (dict(prefix=ODD), MISALIGNED), (dict(ranges=ODD), MISALIGNED)):
        assert f(*{**good, **change}.values(), NULL) == status, change


def test_rotary(b):
    freqs, axis = b.rotary_frequencies(128, (16, 24, 24))
    bad = torch.tensor([1.0, float("inf")] + [0.5] * 62, dtype=torch.float64)

    def call(n=1, tensors=None, x=None, **kw):
        d = dict(rows=10, hdim=128, pairs=64, axes=3, sets=1, in_dtype=1, out_dtype=1, interleaved=0, inverse=0, pad=0,
                 freqs=freqs.data_ptr(), axis=axis.data_ptr(), positions=0x10000)
        d.update(kw)
        t = dict(x=0x10000, y=0x20000, heads=4, pad=0)
        t.update(x or {})
        two = (b.RotaryTensor * 2)(b.RotaryTensor(**t), b.RotaryTensor(**{**t, **(tensors or dict(x=0x30000, y=0x40000))}))
        return b.lib().a2d_rotary(ctypes.byref(b.RotaryDesc(**d)), n, two, NULL)

    for change, status in ((dict(rows=0), INVALID), (dict(rows=(1 << 22) + 1), INVALID), (dict(hdim=72), UNSUPPORTED), (dict(hdim=272), UNSUPPORTED),
                           (dict(pairs=0), INVALID), (dict(pairs=65), INVALID), (dict(axes=0), INVALID), (dict(axes=2), INVALID),
                           (dict(axes=9), INVALID), (dict(sets=0), INVALID), (dict(sets=3), INVALID), (dict(in_dtype=2), UNSUPPORTED),
                           (dict(out_dtype=0), UNSUPPORTED), (dict(interleaved=2), INVALID), (dict(inverse=-1), INVALID), (dict(pad=1), INVALID),
                           (dict(freqs=bad.data_ptr()), INVALID), (dict(freqs=None), INVALID), (dict(positions=None), INVALID),
                           (dict(positions=0x10004), MISALIGNED), (dict(n=0), INVALID), (dict(n=3), INVALID),
                           (dict(x=dict(heads=0)), INVALID), (dict(x=dict(heads=65536)), INVALID), (dict(x=dict(x=None)), INVALID),
                           (dict(x=dict(y=0x20008)), MISALIGNED), (dict(x=dict(lx=b.Layout(128, 100))), INVALID),
                           (dict(x=dict(lx=b.Layout(128, 132))), MISALIGNED), (dict(x=dict(ly=b.Layout(128, 1 << 23))), UNSUPPORTED),
                           (dict(in_dtype=0, x=dict(y=0x10000)), INVALID), (dict(x=dict(y=0x10000, ly=b.Layout(128, 512))), INVALID),
                           (dict(n=2, tensors=dict(x=0x10000, y=0x20000)), INVALID), (dict(n=2, tensors=dict(x=0x30000, y=0x10000)), INVALID)):
        assert call(**change) == status, change


def test_frequencies(b):
    for sections in ((), (0,), (-1, 5), (40, 30)):
        with pytest.raises(b.A2DError):
            b.rotary_frequencies(128, sections)
    freqs, axis = b.rotary_frequencies(64, (2, 3), base=100.0)
    assert freqs.tolist() == [100.0 ** (-2.0 * p / 64) for p in range(5)] and axis.tolist() == [0, 0, 1, 1, 1]
    assert b.rotary_frequencies(64, (2, 2), base=100.0, restart=True)[0].tolist() == [1.0, 100.0 ** -0.5] * 2


def test_tensors_of_the_host_are_refused(b):
    t = torch.zeros(2, 16, 64, dtype=torch.bfloat16)
    r, z = torch.zeros(16, 2, dtype=torch.int32), torch.zeros(2, 16)
    freqs, axis = b.rotary_frequencies(64, (32,))
    for call in (lambda: b.partial_fwd_scored(t, t, t, softcap=1.0), lambda: b.partial_bwd_scored(t, t, t, t, t, z),
                 lambda: b.document_ranges(torch.zeros(2, dtype=torch.int32), 16), lambda: b.rotary(t, r[:, :1].t(), freqs, axis)):
        with pytest.raises(b.A2DError):
            call()


def test_structures(b, tmp_path):
    """The ctypes mirrors against what the C compiler makes of include/a2d.h."""
    code = '#include <stdio.h>\n#include <stddef.h>\n#include "a2d.h"\nint main(void) {\n'
    want = []
    for name, s in (("a2d_score_rules", b.ScoreRules), ("a2d_rotary_desc", b.RotaryDesc), ("a2d_rotary_tensor", b.RotaryTensor)):
        code += '  printf("%%zu ", sizeof(%s));\n' % name
        want.append(ctypes.sizeof(s))
        for field, _ in s._fields_:
            code += '  printf("%%zu ", offsetof(%s, %s));\n' % (name, field)
            want.append(getattr(s, field).offset)
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text(code + "  return 0;\n}\n")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", inc, str(src), "-o", str(exe)], check=True)
    assert [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want
