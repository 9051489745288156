"""Walks are shared where the merge of their parts is one launch: fewer than 2^24 workgroups of eight rows."""
import ctypes

import pytest

from paper_2503_15758_amd import binding as a2d

pytestmark = pytest.mark.gpu
P = 1 << 20                     # some address; never followed


@pytest.mark.parametrize("sequences, kv_heads, group, rows, shared", [
    (8, 8, 4, 1, True), (1, 1, 1, 300, True),
    (65535, 1, 1, 1, True), (65535, 31, 1, 64, True),       # 16.25 million workgroups of the merge
    (65535, 32, 1, 65, False), (65535, 240, 8, 8, False),
])
def test_what_is_shared(sequences, kv_heads, group, rows, shared):
    cache = a2d.CacheDesc(format=a2d.CACHE_E4M3, kv_heads=kv_heads, hdim=128, page_rows=16, pages=4, sequences=sequences, max_pages=64, pad=0,
                          K=P, V=2 * P, K_scales=3 * P, V_scales=4 * P, table=5 * P)
    d = a2d.CachedDesc(heads=kv_heads * group, rows=rows, max_tokens=0, scale=0.1, lens=6 * P, masks=None)
    need = a2d.lib().a2d_cached_workspace_bytes(ctypes.byref(cache), ctypes.byref(d))
    assert (need > 0) == shared
