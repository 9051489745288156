"""The paged cache: written, read back; the ancestors of drafted tokens."""
import math

import pytest
import torch

import cached_reference as ref
from paper_2503_15758_amd import binding as a2d

pytestmark = pytest.mark.gpu

FORMATS = {"bf16": a2d.CACHE_BF16, "e4m3": a2d.CACHE_E4M3, "e2m1": a2d.CACHE_E2M1}


def _tables(gen, sequences, columns, pages):
    assert sequences * columns <= pages
    return torch.randperm(pages, generator=gen)[:sequences * columns].view(sequences, columns).int()


def _expected(old, table, K, starts, index, page_rows, fmt):
    """What the cache's K (codes, scales) is after a write, from what it was."""
    codes, scales = (x.cpu().clone() for x in old)
    n, heads, rows, H = K.shape
    if fmt == "bf16":
        new = K.cpu().bfloat16()
    else:
        c, e = ref.quantised(K.cpu(), fmt)
        new = c.to(torch.uint8) if fmt == "e4m3" else (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8)
        e = (e + 127).to(torch.uint8)
    for b in range(n):
        for j in range(index.shape[1]):
            r, t = int(index[b, j]), int(starts[b]) + j
            if not 0 <= r < rows or not 0 <= t < table.shape[1] * page_rows:
                continue
            page = int(table[b, t // page_rows])
            if not 0 <= page < codes.shape[0]:
                continue
            codes[page, :, t % page_rows] = new[b, :, r]
            if fmt != "bf16":
                scales[page, :, t % page_rows, :e.shape[-1]] = e[b, :, r]
    return codes, scales


def _raw(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)


def _check_write(cache, table, K, V, starts, index, fmt):
    page_rows = cache[0].shape[2]
    all_rows = torch.arange(K.shape[2]).expand(K.shape[0], -1)
    before = [(_raw(cache[i]).clone(), cache[2 + i].clone() if fmt != "bf16" else torch.zeros(1)) for i in range(2)]
    a2d.cache_write(cache, table.cuda(), K, V, starts.cuda(), index.cuda() if index is not None else None)
    for i, x in enumerate((K, V)):
        codes, scales = _expected((before[i][0].view(cache[i].dtype).view(torch.uint8) if fmt != "bf16" else before[i][0].view(torch.bfloat16),
                                   before[i][1]), table, x, starts, index if index is not None else all_rows, page_rows, fmt)
        assert torch.equal(_raw(cache[i]).cpu(), _raw(codes)), "%s of %s" % ("KV"[i], fmt)
        if fmt != "bf16":
            assert torch.equal(cache[2 + i].cpu(), scales)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("H", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, heads, page_rows", [(1, 3, 16), (37, 2, 48), (100, 1, 16)])
def test_write(fmt, H, dtype, rows, heads, page_rows):
    gen = torch.Generator().manual_seed(H + rows)
    n, columns = 3, 1 + (rows + 60) // page_rows
    cache = a2d.cache_empty(3 * columns + 2, heads, page_rows, H, FORMATS[fmt])
    for x in cache:
        _raw(x).fill_(77)
    table = _tables(gen, n, columns, 3 * columns + 2)
    K, V = (torch.randn(n, heads, rows, H, generator=gen).to(dtype).cuda() for _ in range(2))
    starts = torch.tensor([0, 15, 41], dtype=torch.int32)
    _check_write(cache, table, K, V, starts, None, fmt)


@pytest.mark.parametrize("fmt", list(FORMATS))
def test_write_chosen_rows_of_views(fmt):
    """An index that leaves out, repeats and names no rows; tokens outside the table and on no page; K and V as a model keeps them."""
    gen = torch.Generator().manual_seed(1)
    n, heads, rows, H, page_rows = 4, 2, 9, 80, 16
    cache = a2d.cache_empty(20, heads, page_rows, H, FORMATS[fmt])
    for x in cache:
        _raw(x).fill_(7)
    table = _tables(gen, n, 3, 20)
    table[1, 1] = -1
    table[2, 0] = 20
    packed = torch.randn(n, rows, 3, heads, H, generator=gen).bfloat16().cuda()
    K, V = packed[:, :, 1].permute(0, 2, 1, 3), packed[:, :, 2].permute(0, 2, 1, 3)
    index = torch.tensor([[0, 3, 3, 8, -1, 9], [8, 7, 6, 5, 4, 3], [0, 1, 2, 3, 4, 5], [-5, 2 ** 31 - 1, 1, -2 ** 31, 0, 2]], dtype=torch.int32)
    starts = torch.tensor([44, 13, 13, -2], dtype=torch.int32)
    _check_write(cache, table, K, V, starts, index, fmt)
    _check_write(cache, table, K, V, torch.tensor([2 ** 31 - 1, -2 ** 31, 48, 47], dtype=torch.int32), index, fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_every_rounding(fmt):
    """All bf16 numbers, each beside one that sets the scale; ties and their neighbours in fp32; the ends of the range."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    every = every[torch.isfinite(every)].float()
    worth = torch.tensor(ref.code_values(fmt))
    ties = (worth[1:] + worth[:-1]) / 2
    ties = torch.cat([ties, torch.nextafter(ties, torch.zeros(1)), torch.nextafter(ties, torch.full((1,), 1e9)), worth])
    ties = torch.cat([torch.ldexp(ties, torch.tensor(e)) for e in (0, 1, 40, -40, -90, -100, 118)])
    ties = ties[torch.isfinite(ties)]
    values = torch.cat([every, ties, -ties])
    H, heads = 64, 1
    rows = []
    for v, lead in ((values, 0.0), (values, None), (values, 2.0 ** -60), (ties, float(worth[-1]))):
        x = torch.zeros(v.numel(), H)
        x[:, 5] = v
        x[:, 31] = lead if lead is not None else v * 3
        x[:, 32] = v * 0.37
        x[:, 40] = -v
        rows.append(x)
    x = torch.cat(rows)
    x = x[torch.isfinite(x).all(1)]
    pages = -(-x.shape[0] // 4096)
    K = x.view(1, 1, -1, H).cuda()
    cache = a2d.cache_empty(pages, heads, 4096, H, FORMATS[fmt])
    table = torch.arange(pages, dtype=torch.int32).view(1, -1)
    a2d.cache_write(cache, table.cuda(), K, K, torch.zeros(1, dtype=torch.int32).cuda())
    codes, e = ref.quantised(x, fmt)
    got = cache[0].view(torch.uint8).cpu().reshape(-1, cache[0].shape[-1])[:x.shape[0]].long()
    if fmt == "e2m1":
        got = torch.stack([got & 15, got >> 4], -1).flatten(-2)
    assert torch.equal(cache[2].cpu().reshape(-1, 4)[:x.shape[0], :2].long() - 127, e)
    assert torch.equal(got, codes)
    back, _ = a2d.cache_read(cache, table.cuda(), torch.tensor([x.shape[0]], dtype=torch.int32).cuda(), x.shape[0], out_dtype=torch.float32)
    want = ref.decoded(codes, e, fmt).float()
    assert torch.equal(back[0, 0].cpu(), want)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("H", [64, 80, 128])
def test_blocks_that_are_not_finite(fmt, H):
    x = torch.randn(1, 1, 16, H, generator=torch.Generator().manual_seed(3))
    x[0, 0, 0, 3] = math.nan
    x[0, 0, 1, H - 1] = math.inf
    x[0, 0, 2, 33] = -math.inf
    x[0, 0, 3] = 0
    cache = a2d.cache_empty(1, 1, 16, H, FORMATS[fmt])
    table = torch.zeros(1, 1, dtype=torch.int32)
    _check_write(cache, table, x.cuda(), -x.cuda(), torch.zeros(1, dtype=torch.int32), None, fmt)
    K, V = a2d.cache_read(cache, table.cuda(), torch.full((1,), 16, dtype=torch.int32).cuda(), 16)
    for y in (K[0, 0].cpu(), V[0, 0].cpu()):
        blocks = torch.nn.functional.pad(torch.isnan(y).float(), (0, -H % 32)).unflatten(-1, (-1, 32))
        bad = blocks.amax(-1) > 0
        want = torch.zeros_like(bad)
        want[0, 0] = want[1, -1] = want[2, 1] = True
        assert torch.equal(bad, want)
        assert torch.isnan(y[0, :32]).all() and torch.isnan(y[1, (H - 1) // 32 * 32:]).all() and torch.isnan(y[2, 32:64]).all()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("H", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read(fmt, H, dtype):
    gen = torch.Generator().manual_seed(H)
    n, heads, page_rows, columns, rows, first = 4, 2, 48, 4, 67, 29
    cache = ref.new_cache(gen, a2d, fmt, n * columns, heads, page_rows, H)
    table = _tables(gen, n, columns, n * columns)
    table[3, 1] = -7
    lens = torch.tensor([190, 50, 0, 2000], dtype=torch.int32)
    out = [torch.full((n, rows + 2, heads, H), 5.0, dtype=dtype, device="cuda") for _ in range(2)]
    views = [x[:, 1:-1].permute(0, 2, 1, 3) for x in out]
    got = a2d.cache_read(cache, table.cuda(), lens.cuda(), rows, first=first, out=views)
    plain = a2d.cache_read(cache, table.cuda(), lens.cuda(), rows, first=first, out_dtype=dtype)
    for i in range(2):
        values = ref.cache_values(cache, i)
        want = torch.zeros(n, heads, rows, H, dtype=torch.float64)
        for b in range(n):
            end = min(int(lens[b]), columns * page_rows, first + rows)
            if end > first:
                want[b, :, :end - first] = ref.sequence(values, table, b, end)[:, first:].nan_to_num(0.0)
        assert torch.equal(got[i].cpu().double(), want) and torch.equal(plain[i].cpu().double(), want)
        assert got[i].data_ptr() == views[i].data_ptr()
        assert bool((out[i][:, 0] == 5).all()) and bool((out[i][:, -1] == 5).all())


@pytest.mark.parametrize("rows", [1, 2, 7, 63, 64, 65, 130, 256])
@pytest.mark.parametrize("kind", ["random", "chain", "star", "padded"])
def test_tree_masks(rows, kind):
    gen = torch.Generator().manual_seed(rows)
    n = 3
    p = torch.full((n, rows), -1, dtype=torch.int32)
    for b in range(n):
        for i in range(1, rows):
            r = int(torch.randint(-1, i, (1,), generator=gen))
            p[b, i] = {"random": r, "chain": i - 1, "star": 0 if b else -1, "padded": r if r % 3 else [-2, i, i + 5, 2 ** 31 - 1, -2 ** 31][r % 5]}[kind]
    lens = torch.tensor([0, 100000, -5], dtype=torch.int32)
    for given in (lens, None):
        masks, positions = a2d.tree_masks(p.cuda(), given.cuda() if given is not None else None)
        for b in range(n):
            seen = ref.ancestors(p[b].tolist())
            assert masks[b].cpu().tolist() == ref.mask_words(seen, -(-rows // 64))
            base = max(int(lens[b]), 0) if given is not None else 0
            assert positions[b, 0].cpu().tolist() == [base + len(s) - 1 if s else 0 for s in seen]
