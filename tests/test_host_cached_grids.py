"""Calls whose grid passes the 2^32 threads of a launch are refused before anything goes out; without a device."""
import ctypes

import pytest

from paper_2503_15758_amd import binding as a2d
from test_host_cached import UNSUPPORTED, _attend, _cache, _desc


def _call(kv_heads, heads, rows, tokens=16, sequences=65535, **more):
    cache = _cache(sequences=sequences, kv_heads=kv_heads, pages=4, page_rows=16, max_pages=tokens // 16)
    status = _attend(cache, _desc(heads=heads, rows=rows, masks=None), **more)
    return status, a2d.lib().a2d_last_error().decode()


@pytest.mark.parametrize("kv_heads, heads, rows", [
    (257, 257, 1),              # 2^24 walks of 256 threads and more
    (257, 1028, 4), (300, 300, 100),
    (129, 129, 129),            # 2^23 of 512
])
@pytest.mark.parametrize("flags", [0, a2d.TILE_NORMALISED])
@pytest.mark.parametrize("tokens", [16, 1024])
def test_too_many_walks(kv_heads, heads, rows, flags, tokens):
    status, said = _call(kv_heads, heads, rows, tokens, flags=flags)
    assert status == UNSUPPORTED and "threads" in said


def test_too_many_rows_for_the_vector_alu():
    """(a wavefront for each row of each head)"""
    a2d.force_generic(True)
    try:
        status, said = _call(1, 1, 1025, sequences=65535)
    finally:
        a2d.force_generic(False)
    assert status == UNSUPPORTED and "threads" in said


def test_the_workspace_call_says_nothing_about_them():
    cache = _cache(sequences=65535, kv_heads=257, pages=4, page_rows=16, max_pages=1)
    assert a2d.lib().a2d_cached_workspace_bytes(ctypes.byref(cache), ctypes.byref(_desc(heads=257, rows=1, masks=None))) == 0
