"""Refusals of the paged cache's calls, through the C boundary and without a device: every one comes before a launch."""
import ctypes
import math

import pytest
import torch

from paper_2503_15758_amd import binding as a2d

INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = -1, -2, -3, -4
P = 1 << 20                     # some address, 16-byte aligned; never followed


def _cache(**more):
    c = a2d.CacheDesc(format=a2d.CACHE_E4M3, kv_heads=2, hdim=128, page_rows=64, pages=10, sequences=3, max_pages=4, pad=0,
                      K=P, V=2 * P, K_scales=3 * P, V_scales=4 * P, table=5 * P)
    for k, v in more.items():
        setattr(c, k, v)
    return c


def _layout(*strides):
    return a2d.BatchLayout(*(strides or (0, 0, 0)))


BAD_CACHES = [
    (dict(format=3), UNSUPPORTED), (dict(format=-1), UNSUPPORTED), (dict(hdim=72), UNSUPPORTED), (dict(hdim=256), UNSUPPORTED),
    (dict(kv_heads=0), INVALID), (dict(kv_heads=65536), INVALID), (dict(sequences=0), INVALID), (dict(sequences=65536), INVALID),
    (dict(page_rows=0), INVALID), (dict(page_rows=8), INVALID), (dict(page_rows=24), INVALID), (dict(page_rows=(1 << 22) + 16), INVALID),
    (dict(pages=0), INVALID), (dict(pages=1 << 30, page_rows=64), INVALID), (dict(max_pages=0), INVALID),
    (dict(max_pages=(1 << 24) + 1), INVALID), (dict(pad=1), INVALID), (dict(K=0), INVALID), (dict(V=0), INVALID), (dict(table=0), INVALID),
    (dict(K=P + 8), MISALIGNED), (dict(table=P + 4), MISALIGNED), (dict(K_scales=0), INVALID), (dict(V_scales=P + 1), MISALIGNED),
]


def _write(cache=None, rows=5, count=5, dtype=a2d.A2D_BF16, K=P, lk=None, V=2 * P, lv=None, starts=6 * P, index=7 * P):
    return a2d.lib().a2d_cache_write(ctypes.byref(cache or _cache()), rows, count, dtype, K, ctypes.byref(lk or _layout()), V,
                                     ctypes.byref(lv or _layout()), starts, index, None)


def _read(cache=None, lens=6 * P, first=0, rows=5, dtype=a2d.A2D_BF16, K=P, lk=None, V=2 * P, lv=None):
    return a2d.lib().a2d_cache_read(ctypes.byref(cache or _cache()), lens, first, rows, dtype, K, ctypes.byref(lk or _layout()), V,
                                    ctypes.byref(lv or _layout()), None)


def _desc(**more):
    d = a2d.CachedDesc(heads=8, rows=5, max_tokens=0, scale=0.1, lens=6 * P, masks=7 * P)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def _attend(cache=None, d=None, flags=a2d.TILE_NORMALISED, Q=P, K=2 * P, V=3 * P, out0=8 * P, out1=9 * P, out2=10 * P, ws=None, bytes=0):
    return a2d.lib().a2d_partial_fwd_cached(ctypes.byref(cache or _cache()), ctypes.byref(d or _desc()), flags, Q, K, V, out0, out1, out2,
                                            ws, bytes, None)


@pytest.mark.parametrize("bad, status", BAD_CACHES)
def test_caches(bad, status):
    for call in (_write, _read, _attend):
        assert call(_cache(**bad)) == status, call
        assert a2d.lib().a2d_last_error()
    assert a2d.lib().a2d_cached_workspace_bytes(ctypes.byref(_cache(**bad)), ctypes.byref(_desc())) == 0
    assert a2d.lib().a2d_cache_write(None, 1, 1, 1, P, ctypes.byref(_layout()), P, ctypes.byref(_layout()), P, None, None) == INVALID


@pytest.mark.parametrize("bad, status", [
    (dict(rows=0), INVALID), (dict(rows=(1 << 22) + 1), INVALID), (dict(count=0), INVALID), (dict(count=(1 << 22) + 1), INVALID),
    (dict(count=4, index=None), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(K=0), INVALID), (dict(V=P + 4), MISALIGNED),
    (dict(starts=0), INVALID), (dict(index=P + 4), MISALIGNED), (dict(lk=_layout(640, 128, 64)), INVALID),
    (dict(lk=_layout(0, 128, 128)), INVALID), (dict(lv=_layout(1280, 132, 128)), MISALIGNED), (dict(cache=_cache(V=P)), INVALID),
    (dict(rows=1 << 22, count=1, lk=_layout(1 << 32, 1 << 31, 1024)), UNSUPPORTED), (dict(lk=_layout(1 << 41, 128, 256)), INVALID),
])
def test_writes(bad, status):
    assert _write(**bad) == status


@pytest.mark.parametrize("bad, status", [
    (dict(rows=0), INVALID), (dict(first=-1), INVALID), (dict(lens=0), INVALID), (dict(dtype=7), UNSUPPORTED), (dict(K=2 * P), INVALID),
    # outputs whose rows overlap: heads into rows, sequences into heads
    (dict(lk=_layout(1280, 128, 128)), INVALID), (dict(lv=_layout(640, 640, 128)), INVALID), (dict(lv=_layout(128, 256, 768)), INVALID),
])
def test_reads(bad, status):
    assert _read(**bad) == status


@pytest.mark.parametrize("bad, status", [
    (dict(d=_desc(heads=0)), INVALID), (dict(d=_desc(heads=7)), INVALID), (dict(d=_desc(rows=0)), INVALID), (dict(d=_desc(rows=257)), UNSUPPORTED),
    (dict(d=_desc(rows=(1 << 20) + 1, masks=None)), INVALID), (dict(cache=_cache(kv_heads=1), d=_desc(heads=1024, rows=8192, masks=None)), INVALID),
    (dict(d=_desc(max_tokens=-1)), INVALID), (dict(d=_desc(scale=0.0)), INVALID), (dict(d=_desc(scale=-1.0)), INVALID),
    (dict(d=_desc(scale=math.nan)), INVALID), (dict(d=_desc(scale=math.inf)), INVALID), (dict(d=_desc(scale=2e30)), UNSUPPORTED),
    (dict(d=_desc(lens=None)), INVALID), (dict(d=_desc(masks=P + 8)), MISALIGNED), (dict(flags=a2d.TILE_ACCUMULATE), INVALID), (dict(flags=8), INVALID),
    (dict(K=0), INVALID), (dict(V=0), INVALID), (dict(Q=0), INVALID), (dict(Q=P + 2), MISALIGNED), (dict(out0=0), INVALID), (dict(out1=0), INVALID),
    (dict(flags=0, out2=0), INVALID), (dict(out0=P), INVALID), (dict(out0=9 * P), INVALID), (dict(flags=0, out2=9 * P), INVALID),
    (dict(d=_desc(lq=_layout(128, 0, 128))), INVALID), (dict(d=_desc(lo=_layout(640, 128, 128))), INVALID),
    (dict(cache=_cache(sequences=65535, kv_heads=1024, pages=4, max_pages=1 << 20), d=_desc(heads=1024)), UNSUPPORTED),
])
def test_attention(bad, status):
    assert _attend(**bad) == status


@pytest.mark.parametrize("args, status", [
    ((0, 5, P, P, P, P), INVALID), ((65536, 5, P, P, P, P), INVALID), ((1, 0, P, P, P, P), INVALID), ((1, 257, P, P, P, P), UNSUPPORTED),
    ((1, 5, 0, P, P, P), INVALID), ((1, 5, P, P + 4, P, P), MISALIGNED), ((1, 5, P, None, 0, P), INVALID), ((1, 5, P, None, P, 0), INVALID),
])
def test_trees(args, status):
    assert a2d.lib().a2d_tree_masks(*args, None) == status


def test_tensors_on_the_host_are_refused():
    t = torch.zeros(1, 1, dtype=torch.int32)
    cache = tuple(torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16) for _ in range(2))
    x = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: a2d.cache_write(cache, t, x, x, t[0]), lambda: a2d.cache_read(cache, t, t[0], 1), lambda: a2d.tree_masks(t),
                 lambda: a2d.partial_fwd_cached(x, cache, t, t[0])):
        with pytest.raises(a2d.A2DError) as e:
            call()
        assert e.value.status == INVALID
    with pytest.raises(a2d.A2DError):
        a2d.cache_empty(1, 1, 16, 64, format=9, device="cpu")
    with pytest.raises(TypeError):
        a2d.tree_masks([1])


@pytest.mark.parametrize("format, dtype, columns", [(a2d.CACHE_BF16, torch.bfloat16, 80), (a2d.CACHE_E4M3, torch.float8_e4m3fn, 80),
                                                    (a2d.CACHE_E2M1, torch.uint8, 40)])
def test_tensors_of_a_cache(format, dtype, columns):
    c = a2d.cache_empty(3, 2, 32, 80, format, device="cpu")
    assert len(c) == (2 if format == a2d.CACHE_BF16 else 4)
    assert all(x.dtype == dtype and x.shape == (3, 2, 32, columns) for x in c[:2])
    assert all(x.dtype == torch.uint8 and x.shape == (3, 2, 32, 4) for x in c[2:])
