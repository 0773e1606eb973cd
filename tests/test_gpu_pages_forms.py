"""The kernels of 64 and 128 query rows to a workgroup (and of 64 in fp32) over every layout that the calls take: pages of
any size, dense, packed and padded tensors, shared heads, windows without a causal mask, output on the queries, tables wider
than their sequences are long, entries outside the pool, offsets beyond 32 bits, codes and scales in one record."""
import random

import pytest
import torch

import paper_2505_19602_amd as skv
import pages_util as P
import test_gpu_pages as T

pytestmark = pytest.mark.gpu
DEV, BF16, F32, E4M3 = "cuda", torch.bfloat16, torch.float32, P.E4M3
MASKS = [dict(causal=True), {}, dict(window=37, sinks=3), dict(causal=True, window=300, sinks=70), dict(window=200, sinks=0)]


def _many(rows, new):
    """Lengths and counts of 128 sequences, three of them with rows: units enough for workgroups of many query rows."""
    lens, counts = [0] * 128, [0] * 128
    for s, n, t in zip(T.BUSY, (rows, max(rows - 37, 1), rows), (new, max(new // 2, 1), max(new - 1, 1))):
        lens[s], counts[s] = n, min(n, t)
    return lens, counts


def _run(shape, pages, q, out, new, causal=False, window=0, sinks=0, **chunk):
    mask = dict(causal=causal, window=window, n_sink=sinks)
    ws = torch.full((skv.pages_workspace_bytes(shape, pages, new, **mask),), 255, dtype=torch.uint8, device=DEV)
    skv.pages_attend(shape, pages, q, out, ws, max_new=new, **mask, **chunk)
    torch.cuda.synchronize()
    return ws.numel()


def _compare(cache, s, q, have, causal=False, window=0, sinks=0):
    want, tol = P.attend(cache, s, q, causal, window, sinks, cache.d ** -0.5)
    err = (have.cpu().double() - want).abs()
    assert torch.all(err <= tol), f"sequence {s}: {float((err / tol).max()):.3g} of the bound"


# (rows of a page, packed, query rows of a unit, cached rows): 64 and 128 rows to a workgroup, not multiples of them
LAYOUTS = [(64, False, 100, 200), (256, True, 300, 333), (128, False, 290, 700), (32, True, 90, 129)]


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4, 5, 8])
def test_layouts_and_shared_heads_of_many_rows(dtype, cache_dtype, d, group):
    for i, (page, packed, unit_rows, rows) in enumerate(LAYOUTS):
        for mask in (MASKS[(i + group) % 5], MASKS[(i + group + 2) % 5]):
            new = -(-unit_rows // group)
            print(f"layouts {dtype} {cache_dtype} d {d} group {group} page {page} packed {packed} new {new} rows {rows} {mask}",
                  flush=True)
            lens, counts = _many(rows, new)
            T._check_lengths(10 * i + group, lens, counts, 2 * group, 2, d, dtype, cache_dtype, page, new, packed=packed, **mask)


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
@pytest.mark.parametrize("mask", MASKS)
def test_tables_wider_than_the_sequences_are_long(dtype, cache_dtype, mask):
    # few sequences under tables for 131072 rows, as a captured call has them: row groups and cuts follow the table's width
    for d, page, group, new, lens, counts in ((128, 16, 4, 64, [600, 64, 0], [64, 50, 0]), (64, 256, 1, 200, [600, 200, 5], [200, 1, 5]),
                                              (128, 64, 8, 20, [2100, 20, 333], [20, 20, 7])):
        print(f"wide table {dtype} {cache_dtype} d {d} page {page} group {group} new {new} {mask}", flush=True)
        T._check_lengths(new, lens, counts, 2 * group, 2, d, dtype, cache_dtype, page, new, packed=page == 64,
                         width=131072 // page, **mask)


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_output_on_the_queries(dtype, cache_dtype, d):
    for new, group, page, mask in ((33, 3, 64, MASKS[0]), (60, 5, 32, MASKS[3]), (3, 8, 128, MASKS[0])):
        lens, counts = _many(250, new)
        cache = P.Cache(new, lens, 2, d, page, cache_dtype, dtype)
        shape = skv.Shape(128, 2 * group, d, dtype)
        q, take, chunk = T._tokens(new, 128, 2 * group, counts, new, d, dtype, False)
        on = q.to(DEV)
        _run(shape, cache.on(DEV), on, on, new, first=None, count=chunk["count"], **mask)
        got, same = on.cpu(), torch.ones(q.shape, dtype=torch.bool)
        for s in T.BUSY:
            _compare(cache, s, take(q, s), take(got, s), **mask)
            take(same, s)[:] = False
        assert torch.equal(got[same], q[same]), "rows behind a sequence's last token were written"


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
@pytest.mark.parametrize("new", [1, 40, 150])
def test_padded_batches_and_token_major_tensors(dtype, cache_dtype, new):
    # tokens at the END of each sequence's rows (padded on the left); q, k and v in one token-major tensor; written and attended
    d, group, page = 64, 2, 64
    lens, counts = _many(max(new, 170), new)
    heads = 2 * group
    cache = P.Cache(new, lens, 2, d, page, cache_dtype, dtype)
    shape, pages = skv.Shape(128, heads, d, dtype), cache.on(DEV)
    fused = torch.randn(128, new, heads + 4, d, generator=torch.Generator().manual_seed(new)).to(dtype)
    q, k, v = (fused.to(DEV)[:, :, a:b].transpose(1, 2) for a, b in ((0, heads), (heads, heads + 2), (heads + 2, None)))
    first = torch.tensor([new - n for n in counts], dtype=torch.int32, device=DEV)
    count = torch.tensor(counts, dtype=torch.int32, device=DEV)
    skv.pages_write(shape, pages, k, v, first=first, count=count)
    out = torch.full((128, heads, new, d), 7.0, dtype=dtype, device=DEV)
    _run(shape, pages, q, out, new, causal=True, first=first, count=count)
    skv.pages_check(shape, pages, cache.table.tolist(), lens, first=first.tolist(), count=counts, max_new=new, n_row=new)
    for name in ("k", "v"):
        cache.pool[name] = getattr(pages, name).cpu()
        if cache_dtype == E4M3:
            cache.scales[name] = getattr(pages, name + "_scale").cpu()
    for s in T.BUSY:
        at = slice(new - counts[s], new)
        for name, a in (("k", heads), ("v", heads + 2)):
            rows = fused[s, at, a:a + 2].transpose(0, 1)
            if cache_dtype == E4M3:
                codes, scale = P.quantised_tensor(rows)
                rows = codes.float().double() * torch.ldexp(torch.ones(()).double(), scale.int() - 127).unsqueeze(-1)
            assert torch.equal(cache.rows(name, s)[:, lens[s] - counts[s]:], rows.double())
        _compare(cache, s, fused[s, at, :heads].transpose(0, 1), out[s, :, at], causal=True)
        assert torch.all(out[s, :, :new - counts[s]] == 7.0)
    assert all(torch.all(out[s] == 7.0) for s in range(128) if s not in T.BUSY)


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
@pytest.mark.parametrize("mask", MASKS[:4])
def test_entries_outside_the_pool_read_as_zeros(dtype, cache_dtype, mask):
    for d, page, new, rows in ((128, 16, 80, 333), (64, 64, 150, 333), (128, 32, 150, 2500)):
        def change(cache):
            used = -(-rows // page)
            for s, bad in zip(T.BUSY, (-1, cache.pool["k"].shape[0], 2 ** 31 - 1)):
                n = -(-cache.lens[s] // page)
                for x in {0, n // 2, n - 1}:
                    cache.table[s, x] = bad
        lens, counts = _many(rows, new)
        T._check_lengths(rows + page, lens, counts, 2, 2, d, dtype, cache_dtype, page, new, packed=page == 64, change=change, **mask)


def _records(n_page, heads, page, d, dtype, cache_dtype):
    """A pool as one tensor: keys, values and scales of a page behind each other, `n_page` such records.  Views of them."""
    e = torch.zeros((), dtype=cache_dtype).element_size()
    unit = heads * page * d * e
    record = 2 * unit + (2 * heads * page if cache_dtype == E4M3 else 16)
    flat = torch.zeros(n_page * record, dtype=torch.uint8, device=DEV)
    typed = flat.view(cache_dtype)
    pools = [typed.as_strided((n_page, heads, page, d), (record // e, page * d, d, 1), i * unit // e) for i in range(2)]
    scales = [None, None]
    if cache_dtype == E4M3:
        scales = [flat.as_strided((n_page, heads, page), (record, page, 1), 2 * unit + i * heads * page) for i in range(2)]
    return flat, pools, scales


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
@pytest.mark.parametrize("new", [1, 80, 150])
def test_records_beyond_32_bit_offsets(dtype, cache_dtype, new):
    # the pages of three sequences are the last of 4.3 GB, keys, values and scales of a page in one record
    d, heads, page, rows = 128, 2, 64, 200
    lens, counts = _many(rows, new)
    cache = P.Cache(new, lens, heads, d, page, cache_dtype, dtype)
    few = cache.pool["k"].shape[0]
    e = torch.zeros((), dtype=cache_dtype).element_size()
    n_page = (1 << 32) // (2 * heads * page * d * e) + few
    flat, pools, scales = _records(n_page, heads, page, d, dtype, cache_dtype)
    at = n_page - few
    assert at * (flat.numel() // n_page) > 4 * 10 ** 9 and flat.numel() > 1 << 32
    for i, name in enumerate(("k", "v")):
        pools[i][at:].view(torch.uint8 if e == 1 else pools[i].dtype).copy_(
            cache.pool[name].view(torch.uint8 if e == 1 else pools[i].dtype).to(DEV))
        if scales[i] is not None:
            scales[i][at:] = cache.scales[name].to(DEV)
    table = torch.where(cache.table >= 0, cache.table + at, -1).to(DEV)
    pages = skv.Pages(*pools, table, torch.tensor(lens, dtype=torch.int32, device=DEV), *scales)
    shape = skv.Shape(128, 2 * heads, d, dtype)
    # written first, so that all three calls go through the records
    k, take, chunk = T._tokens(1, 128, heads, counts, new, d, dtype, True)
    v = T._tokens(2, 128, heads, counts, new, d, dtype, True)[0]
    before = flat[:1 << 20].clone()
    skv.pages_write(shape, pages, k.to(DEV), v.to(DEV), **chunk)
    for s in T.BUSY:
        for t in range(counts[s]):
            r = lens[s] - counts[s] + t
            place = int(cache.table[s, r // page]), slice(None), r % page
            for name, x in (("k", k), ("v", v)):
                row = take(x, s)[:, t]
                if cache_dtype == E4M3:
                    codes, cache.scales[name][place] = P.quantised_tensor(row)
                    cache.pool[name].view(torch.uint8)[place] = codes.view(torch.uint8)
                else:
                    cache.pool[name][place] = row
    bits = lambda t: t.contiguous().view(torch.uint8).cpu()
    for i, name in enumerate(("k", "v")):
        assert torch.equal(bits(pools[i][at:]), bits(cache.pool[name]))
        assert scales[i] is None or torch.equal(scales[i][at:].cpu(), cache.scales[name])
    assert torch.equal(flat[:1 << 20], before)
    q, take, chunk = T._tokens(3, 128, 2 * heads, counts, new, d, dtype, True)
    out = torch.full(q.shape, 7.0, dtype=dtype, device=DEV)
    _run(shape, pages, q.to(DEV), out, new, causal=True, first=chunk["first"], count=chunk["count"])
    back = torch.full((2, 128, 2 * heads, rows, d), 7.0, dtype=dtype, device=DEV)
    skv.pages_read(shape, pages, None, rows, back[0], back[1])
    torch.cuda.synchronize()
    for s in T.BUSY:
        _compare(cache, s, take(q, s), take(out, s), causal=True)
        for i, name in enumerate(("k", "v")):
            assert torch.equal(back[i, s, :, :lens[s]].cpu().double(), cache.rows(name, s).repeat_interleave(2, 0))
            assert torch.all(back[i, s, :, lens[s]:] == 7.0)


@pytest.mark.parametrize("dtype,cache_dtype", T.TYPES)
def test_rows_of_out_that_lie_between_each_other(dtype, cache_dtype):
    # no dimension of the output holds another whole: heads 3 rows apart, tokens 2
    d, new = 64, 4
    cache = P.Cache(1, [77], 2, d, 16, cache_dtype, dtype)
    q = torch.randn(1, 2, new, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    flat = torch.full((10, d), 7.0, dtype=dtype, device=DEV)
    out = flat.as_strided((1, 2, new, d), (10 * d, 3 * d, 2 * d, 1))
    _run(skv.Shape(1, 2, d, dtype), cache.on(DEV), q.to(DEV), out, new, causal=True)
    _compare(cache, 0, q[0], out[0], causal=True)
    assert torch.all(flat[[1, 8]] == 7.0)
    with pytest.raises(skv.ScaleKVError, match="coincide"):
        _run(skv.Shape(1, 2, d, dtype), cache.on(DEV), q.to(DEV), flat.as_strided((1, 2, new, d), (10 * d, 2 * d, 2 * d, 1)), new)


def test_the_binding_refuses_lengths_and_rows_that_do_not_fit_each_other():
    S, H, d, dtype = 2, 4, 64, BF16
    shape, pages = skv.Shape(S, H, d, dtype), P.Cache(1, [20, 30], 2, d, 16, E4M3, dtype).on(DEV)
    rows = lambda n, h: torch.zeros(n, h, d, dtype=dtype, device=DEV)
    ws = torch.empty(skv.pages_workspace_bytes(shape, pages, 3), dtype=torch.uint8, device=DEV)
    first = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    bits = [t.view(torch.uint8).clone() for t in (pages.k, pages.v)]
    for a, b in ((6, 4), (4, 6), (6, 0)):
        with pytest.raises(skv.ScaleKVError, match=f"k_new has {a} rows and v_new {b}"):
            skv.pages_write(shape, pages, rows(a, 2), rows(b, 2), first=first, max_new=3)
        with pytest.raises(skv.ScaleKVError, match=f"q has {a} rows and out {b}"):
            skv.pages_attend(shape, pages, rows(a, H), rows(b, H), ws, first=first, max_new=3)
    torch.cuda.synchronize()
    assert all(torch.equal(x, t.view(torch.uint8)) for x, t in zip(bits, (pages.k, pages.v)))
    table = pages.table.tolist()
    skv.pages_check(shape, pages, table, [20, 30], first=[0, 3], max_new=3, n_row=6, packed=True)
    with pytest.raises(skv.ScaleKVError, match="sequences 0 and 1 share row 2"):
        skv.pages_check(shape, pages, table, [20, 30], first=[0, 2], max_new=3, n_row=6, packed=True)
