"""a2d_partial_fwd_cached through the C boundary, for what the calls on tensors leave to the library: a workspace or none."""
import ctypes

import torch

from paper_2503_15758_amd import binding as a2d

FORMATS = {torch.bfloat16: a2d.CACHE_BF16, torch.float8_e4m3fn: a2d.CACHE_E4M3, torch.uint8: a2d.CACHE_E2M1}


def _ptr(t):
    return None if t is None else t.data_ptr()


def without_workspace(x, normalised=False, max_tokens=0):
    """The outputs for a problem of test_gpu_cached_attention.py's kind, each walk in one workgroup."""
    held = {k: None if x[k] is None else x[k].cuda().contiguous() for k in ("Q", "K", "V", "masks", "table", "lens")}
    n, heads, rows, H = held["Q"].shape
    cache = list(x["cache"]) + [None] * (4 - len(x["cache"]))
    pages, kv_heads, page_rows = cache[0].shape[:3]
    c = a2d.CacheDesc(FORMATS[cache[0].dtype], kv_heads, H, page_rows, pages, n, held["table"].shape[1], 0, *(_ptr(t) for t in cache),
                      held["table"].data_ptr())
    d = a2d.CachedDesc(heads=heads, rows=rows, max_tokens=max_tokens, scale=x["scale"], lens=held["lens"].data_ptr(), masks=_ptr(held["masks"]))
    out = [torch.empty(n, heads, rows, H, device="cuda", dtype=torch.bfloat16 if normalised else torch.float32)]
    out += [torch.empty(n, heads, rows, device="cuda") for _ in range(1 if normalised else 2)]
    status = a2d.lib().a2d_partial_fwd_cached(ctypes.byref(c), ctypes.byref(d), a2d.TILE_NORMALISED if normalised else 0, _ptr(held["Q"]),
                                              _ptr(held["K"]), _ptr(held["V"]), *(ctypes.c_void_p(_ptr(t)) for t in out),
                                              *([None] if normalised else []), None, 0, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert status == 0, a2d.lib().a2d_last_error()
    torch.cuda.synchronize()
    return tuple(out)
