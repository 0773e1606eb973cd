"""The paged cache on the GPU: rows written and read back bit for bit, attention over the pages against 64 bits, with
bounds derived in pages_util.attend."""
import math
import random

import numpy as np
import pytest
import torch

import paper_2505_19602_amd as skv
import pages_util as P

pytestmark = pytest.mark.gpu
DEV, BF16, F32, E4M3 = "cuda", torch.bfloat16, torch.float32, P.E4M3


def _tokens(seed, seqs, heads, counts, new, d, dtype, packed, scale=1.0):
    """Rows of new tokens on the device, a function that takes one sequence's [heads, n, d], first and count tensors."""
    g = torch.Generator().manual_seed(seed)
    if packed:
        total = sum(counts)
        x = (torch.randn(max(total, 1), heads, d, generator=g) * scale).to(dtype)
        first = [sum(counts[:s]) for s in range(seqs)]
        take = lambda t, s: t[first[s]:first[s] + counts[s]].transpose(0, 1)
        firsts = torch.tensor(first, dtype=torch.int32, device=DEV)
    else:
        x = (torch.randn(seqs, heads, new, d, generator=g) * scale).to(dtype)
        take, firsts = (lambda t, s: t[s, :, :counts[s]]), None
    return x, take, dict(first=firsts, count=torch.tensor(counts, dtype=torch.int32, device=DEV), max_new=new)


def _check_attend(seed, seqs, heads, kv_heads, d, dtype, cache_dtype, page, most, new, *, ragged=False, packed=False,
                  causal=False, window=0, sinks=0, scale=1.0, width=None, change=None, sm_scale=0.0):
    print(f"attend {seqs} seqs {heads}/{kv_heads} heads d {d} {dtype} cache {cache_dtype} page {page} rows {most} new {new} "
          f"ragged {ragged} packed {packed} causal {causal} window {window} sinks {sinks}", flush=True)
    lens, counts = P.lengths(random.Random(seed), seqs, most, new, ragged)
    return _check_lengths(seed, lens, counts, heads, kv_heads, d, dtype, cache_dtype, page, new, packed=packed, causal=causal,
                          window=window, sinks=sinks, scale=scale, width=width, change=change, sm_scale=sm_scale)


def _check_lengths(seed, lens, counts, heads, kv_heads, d, dtype, cache_dtype, page, new, *, packed=False, causal=False, window=0,
                   sinks=0, scale=1.0, width=None, change=None, sm_scale=0.0):
    seqs = len(lens)
    cache = P.Cache(seed, lens, kv_heads, d, page, cache_dtype, dtype, width=width, scale=scale)
    if change:
        change(cache)
    shape = skv.Shape(seqs, heads, d, dtype, sm_scale)
    q, take, chunk = _tokens(seed + 1, seqs, heads, counts, new, d, dtype, packed, scale)
    pages, qd = cache.on(DEV), q.to(DEV)
    out = torch.full_like(qd, 7.0)
    need = skv.pages_workspace_bytes(shape, pages, new, causal=causal, window=window, n_sink=sinks)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)      # (NaN wherever it is read before it is written)
    skv.pages_attend(shape, pages, qd, out, ws, causal=causal, window=window, n_sink=sinks, **chunk)
    torch.cuda.synchronize()
    got, touched = out.cpu(), torch.zeros(out.shape, dtype=torch.bool)
    for s in range(seqs):
        if counts[s] == 0:
            continue
        want, tol = P.attend(cache, s, take(q, s), causal, window, sinks, sm_scale or d ** -0.5)
        have = take(got, s).double()
        same = (have == want) | (have.isnan() & want.isnan())   # infinities and NaN where they belong
        wrong = (~(same | ((have - want).abs() <= tol))).nonzero().tolist()
        assert not wrong, f"sequence {s}: {len(wrong)} elements off: " + ", ".join(
            f"{x}: {have[tuple(x)]:.5g}, want {want[tuple(x)]:.5g} within {tol[tuple(x)]:.2g}" for x in wrong[:4] + wrong[-2:])
        take(touched, s)[:] = True
    assert torch.all(got[~touched] == 7.0), "rows behind a sequence's last token were written"
    return got


def _attend(shape, pages, q, out, new, **kw):
    """pages_attend with a workspace of the size that it asks for."""
    mask = {x: kw[x] for x in ("causal", "window", "n_sink") if x in kw}
    ws = torch.full((skv.pages_workspace_bytes(shape, pages, new, **mask),), 255, dtype=torch.uint8, device=DEV)
    skv.pages_attend(shape, pages, q, out, ws, max_new=new, **kw)


TYPES = [(BF16, BF16), (BF16, E4M3), (F32, F32), (F32, E4M3)]


# ---- writing and reading

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_quantised_rows_are_the_definitions_bit_for_bit(dtype, d):
    # rows of every exponent and of one-sided, constant, zero and non-finite content, through write and read
    g = torch.Generator().manual_seed(d)
    rows = [torch.randn(d, generator=g) * 2.0 ** e for e in range(-126, 128, 3)]
    rows += [torch.full((d,), 448.0 * 2.0 ** e) for e in (-130, -120, -30, 0, 30, 118, 119)]
    rows += [torch.full((d,), math.nextafter(448.0, 449.0)), torch.zeros(d), torch.full((d,), 3.0e38),
             torch.full((d,), -3.3895e38)]
    for value in (math.inf, -math.inf, math.nan):
        x = torch.randn(d, generator=g)
        x[5] = value
        rows += [x, torch.full((d,), value)]
    x = torch.zeros(d)
    x[0], x[1:] = 448.0, torch.arange(1, d) * 2.0 ** -10        # ties and values below the least code
    rows.append(x)
    x = torch.stack(rows).clamp(-3.3895e38, 3.3895e38).where(torch.isfinite(torch.stack(rows)), torch.stack(rows)).to(dtype)
    n = x.shape[0]
    cache = P.Cache(1, [n], 1, d, 16, E4M3, dtype)
    shape, pages = skv.Shape(1, 1, d, dtype), cache.on(DEV)
    new = x.reshape(1, 1, n, d)
    skv.pages_write(shape, pages, new.to(DEV), (-new).to(DEV))
    back = torch.full((2, 1, 1, n + 2, d), 7.0, dtype=dtype, device=DEV)
    skv.pages_read(shape, pages, None, n, back[0], back[1])
    torch.cuda.synchronize()
    assert torch.all(back[:, :, :, n:] == 7.0)
    for i in range(n):
        codes, k = P.quantised(x[i].double().numpy())
        page, slot = int(cache.table[0, i // 16]), i % 16
        for sign, pool, scale, out in ((1, pages.k, pages.k_scale, back[0]), (-1, pages.v, pages.v_scale, back[1])):
            assert int(scale[page, 0, slot]) == k + 127, f"row {i}"
            have = pool[page, 0, slot].float().cpu().double().numpy()
            assert np.array_equal(have, sign * codes, equal_nan=True), f"row {i}"
            value = np.ldexp(sign * codes, k)
            assert np.all(np.isfinite(value) | np.isnan(codes))
            assert np.array_equal(out[0, 0, i].cpu().double().numpy(), value, equal_nan=True), f"row {i}"


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("packed", [False, True])
def test_write_touches_the_new_rows_alone(dtype, cache_dtype, d, page, packed):
    seqs, heads, new = 5, 3, 37
    lens, counts = [37, 300, 64, 5, 0], [37, 1, 17, 0, 0]
    cache = P.Cache(d + page, lens, heads, d, page, cache_dtype, dtype, width=20)
    shape, pages = skv.Shape(seqs, 2 * heads, d, dtype), cache.on(DEV)
    k, take, chunk = _tokens(3, seqs, heads, counts, new, d, dtype, packed)
    v = _tokens(4, seqs, heads, counts, new, d, dtype, packed)[0]
    skv.pages_write(shape, pages, k.to(DEV), v.to(DEV), **chunk)
    torch.cuda.synchronize()
    for s in range(seqs):
        for t in range(counts[s]):
            r = lens[s] - counts[s] + t
            at = int(cache.table[s, r // page]), slice(None), r % page
            for name, x in (("k", k), ("v", v)):
                row = take(x, s)[:, t]
                if cache_dtype == E4M3:
                    codes, scale = P.quantised_tensor(row)
                    cache.pool[name].view(torch.uint8)[at] = codes.view(torch.uint8)
                    cache.scales[name][at] = scale
                else:
                    cache.pool[name][at] = row
    bits = lambda t: t.contiguous().view(torch.uint8)
    for name, have, scale in (("k", pages.k, pages.k_scale), ("v", pages.v, pages.v_scale)):
        assert torch.equal(bits(have.cpu()), bits(cache.pool[name]))
        assert scale is None or torch.equal(scale.cpu(), cache.scales[name])


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d,group", [(64, 1), (128, 3)])
@pytest.mark.parametrize("listed", [False, True])
def test_read_brings_back_what_the_pages_hold(dtype, cache_dtype, d, group, listed):
    seqs, kv_heads, page, n_row = 4, 2, 32, 45
    lens = [45, 33, 0, 100]
    cache = P.Cache(d, lens, kv_heads, d, page, cache_dtype, dtype)
    heads = kv_heads * group
    shape, pages = skv.Shape(seqs, heads, d, dtype), cache.on(DEV)
    idx = None
    if listed:  # places past the end, negative ones and repeated ones among them
        idx = torch.randint(-3, 110, (seqs, heads, n_row), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    roomy = torch.full((2, seqs, heads, n_row + 3, d), 7.0, dtype=dtype, device=DEV)
    skv.pages_read(shape, pages, None if idx is None else idx.to(DEV), n_row, roomy[0], roomy[1])
    torch.cuda.synchronize()
    for i, name in enumerate(("k", "v")):
        have = roomy[i].cpu().double()
        for s in range(seqs):
            rows = cache.rows(name, s)
            for h in range(heads):
                for t in range(n_row + 3):
                    r = -1 if t >= n_row else t if idx is None else int(idx[s, h, t])
                    want = rows[h // group, r] if 0 <= r < lens[s] else torch.full((d,), 7.0).double()
                    assert torch.equal(have[s, h, t], want), (name, s, h, t)


# ---- attention

EDGES = [(1, 1), (1, 15), (1, 16), (1, 17), (1, 63), (1, 64), (1, 65), (1, 127), (1, 129), (1, 255), (1, 257), (1, 700),
         (2, 2), (2, 130), (15, 15), (16, 40), (17, 17), (17, 129), (31, 100), (33, 33), (33, 200), (64, 65), (65, 300),
         (127, 128), (129, 129), (130, 400)]


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_attend_at_the_edges_of_tiles_and_pages(dtype, cache_dtype, d, causal):
    for i, (new, rows) in enumerate(EDGES):
        _check_attend(100 * i + d, 2, 2, 2, d, dtype, cache_dtype, (16, 32, 64, 128, 256)[i % 5], rows, new, causal=causal)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,group", [(1, 1), (1, 4), (1, 8), (1, 20), (1, 40), (3, 5), (5, 8), (9, 16), (40, 2), (150, 1)])
def test_attend_shared_heads_and_ragged_sequences(dtype, cache_dtype, d, new, group):
    for packed in (False, True):
        _check_attend(new * 31 + group, 5, 2 * group, 2, d, dtype, cache_dtype, 16, 170, new, ragged=True, packed=packed,
                      causal=packed)


WINDOWS = [(1, 0, 1, 300), (1, 4, 1, 300), (2, 1, 40, 40), (7, 16, 1, 64), (16, 4, 17, 200), (63, 64, 33, 300), (64, 1, 129, 500),
           (65, 100, 70, 800), (100, 300, 20, 400), (128, 3, 1, 1000), (129, 64, 300, 700), (1000, 5, 9, 500)]


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_attend_windows_and_sinks(dtype, cache_dtype, d, causal):
    for i, (window, sinks, new, rows) in enumerate(WINDOWS):
        _check_attend(10 * i + d, 2, 2, 1, d, dtype, cache_dtype, (16, 64, 256)[i % 3], rows, new, ragged=i % 2 == 1,
                      packed=i % 4 == 1, causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 3000])
def test_attend_long_caches_split_over_workgroups(dtype, cache_dtype, d, window):
    for new, group, rows in ((1, 1, 9000), (1, 8, 5001), (4, 4, 4097), (40, 4, 5000)):
        shape = skv.Shape(2, 2 * group, d, dtype)
        pages = P.Cache(1, [rows, 1], 2, d, 64, cache_dtype, dtype).on(DEV)
        assert skv.pages_workspace_bytes(shape, pages, new, causal=True, window=window, n_sink=9) > 0
        _check_attend(rows, 2, 2 * group, 2, d, dtype, cache_dtype, 64, rows, new, ragged=True, causal=True, window=window,
                      sinks=9)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("scale", [0.01, 6.0])
def test_attend_flat_and_peaked_weights(dtype, cache_dtype, scale):
    for d, new, rows in ((64, 1, 700), (128, 140, 333), (128, 20, 300)):
        _check_attend(int(10 * scale), 2, 4, 2, d, dtype, cache_dtype, 32, rows, new, causal=True, scale=scale)
    _check_attend(3, 2, 4, 2, 64, dtype, cache_dtype, 32, 300, 33, causal=True, sm_scale=0.4)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("new", [1, 20, 150])
def test_attend_scores_that_rise_and_fall(dtype, cache_dtype, new):
    # the largest score sits in the first, a middle or the last row: the running maximum moves at every place
    d = 128
    for where in (0, 31, 32, 64, 150, 299):
        def change(cache):
            for s in range(2):
                for h in range(2):
                    row = torch.full((d,), 3.0)
                    if cache_dtype == E4M3:
                        p, slot = int(cache.table[s, where // 16]), where % 16
                        cache.pool["k"][p, h, slot], cache.scales["k"][p, h, slot] = (row * 2.0 ** 7).to(E4M3), 120
                    else:
                        cache.put("k", s, where, h, row)
        _check_attend(where, 2, 2, 2, d, dtype, cache_dtype, 16, 300, new, scale=2.0, change=change)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window", [0, 5, 40])
def test_what_a_token_does_not_see_does_not_reach_it(dtype, d, value, window):
    # values and keys that are not finite, in rows that some tokens of a tile see and others do not
    for new, rows, group in ((40, 40, 1), (130, 200, 1), (6, 70, 4), (1, 90, 1), (3, 700, 8), (130, 3500, 1), (70, 2500, 1)):
        bad = {0, 3, rows - new + new // 2, rows - 1, rows - 2, max(0, rows - 45)}

        def change(cache):
            for r in bad:
                cache.pool["v"][int(cache.table[0, r // 16]), 0, r % 16, 3::7] = value
            cache.pool["k"][int(cache.table[0, (rows - 1) // 16]), 0, (rows - 1) % 16, 0] = math.nan
            for name in ("k", "v"):             # pages of nobody, and slots behind the last row
                for p in cache.unused:
                    cache.pool[name][p] = math.nan
                if rows % 16:
                    cache.pool[name][int(cache.table[0, rows // 16]), :, rows % 16:] = math.nan
        _check_attend(rows, 1, group, 1, d, dtype, dtype, 16, rows, new, causal=True, window=window, sinks=2, change=change)


@pytest.mark.parametrize("window", [0, 30])
def test_nan_codes_stay_where_they_are_seen(window):
    def change(cache):
        for r in (0, 2, 150, 190):
            p = int(cache.table[0, r // 16])
            cache.pool["v"].view(torch.uint8)[p, 0, r % 16, 1::5] = 0x7f
            cache.pool["v"].view(torch.uint8)[p, 0, r % 16, 2::5] = 0xff
    for dtype in (BF16, F32):
        _check_attend(5, 1, 2, 1, 128, dtype, E4M3, 16, 200, 130, causal=True, window=window, sinks=1, change=change)
        _check_attend(5, 1, 2, 1, 64, dtype, E4M3, 16, 200, 8, causal=True, window=window, sinks=1, change=change)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [{}, dict(causal=True), dict(causal=True, window=37, sinks=3)])
def test_codes_and_scales_that_nobody_wrote_reach_nothing(dtype, d, mask):
    # rows behind the last one and pages of nobody hold NaN codes with the scale byte 255, as memory comes
    for new, rows in ((1, 77), (20, 85), (40, 130), (70, 333), (130, 1300)):
        def change(cache):
            for name in ("k", "v"):
                dead = [(p, 0) for p in cache.unused] + [(int(cache.table[s, rows // 16]), rows % 16) for s in range(2)]
                for p, slot in dead:
                    cache.pool[name].view(torch.uint8)[p, :, slot:] = 0x7f
                    cache.scales[name][p, :, slot:] = 255
        _check_attend(rows, 2, 4, 2, d, dtype, E4M3, 16, rows, new, change=change, **mask)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
def test_tokens_that_see_nothing_get_zeros(dtype, cache_dtype):
    # sequences shorter than their chunk (positions below zero see nothing under a causal mask) and empty ones
    d, new, heads = 64, 9, 2
    shape = skv.Shape(3, heads, d, dtype)
    cache = P.Cache(1, [4, 0, 9], heads, d, 16, cache_dtype, dtype)
    pages = cache.on(DEV)
    q = torch.randn(3, heads, new, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    out = torch.full((3, heads, new, d), 7.0, dtype=dtype, device=DEV)
    _attend(shape, pages, q.to(DEV), out, new, causal=True)
    torch.cuda.synchronize()
    assert torch.all(out[0, :, :5] == 0) and torch.all(out[1] == 0)
    want, tol = P.attend(cache, 0, q[0, :, 5:], True, 0, 0, d ** -0.5)
    assert torch.all((out[0, :, 5:].cpu().double() - want).abs() <= tol)
    want, tol = P.attend(cache, 2, q[2], True, 0, 0, d ** -0.5)
    assert torch.all((out[2].cpu().double() - want).abs() <= tol)


def test_all_scores_minus_infinity_give_zeros_not_nan():
    d, dtype = 64, F32
    cache = P.Cache(1, [70], 1, d, 16, dtype, dtype)
    cache.pool["k"].fill_(-math.inf)
    q = torch.ones(1, 1, 3, d)
    out = torch.full((1, 1, 3, d), 7.0, device=DEV)
    _attend(skv.Shape(1, 1, d, dtype), cache.on(DEV), q.to(DEV), out, 3, causal=True)
    assert torch.all(out == 0)


@pytest.mark.parametrize("dtype,cache_dtype", [(BF16, BF16), (BF16, E4M3), (F32, F32)])
def test_values_out_of_range_lead_nowhere(dtype, cache_dtype):
    # pages that are not in the pool read as zeros and are not written; lengths, counts and rows are brought into range
    d, seqs, heads, page = 64, 3, 2, 16
    cache = P.Cache(1, [50, 64, 64], heads, d, page, cache_dtype, dtype)
    cache.table[0, 1] = -5
    cache.table[1, 2] = cache.pool["k"].shape[0]
    cache.table[2, 0] = 2 ** 31 - 1
    shape, pages = skv.Shape(seqs, heads, d, dtype), cache.on(DEV)
    pages.lens[2] = 10 ** 9                                           # ends with the table: 64 rows
    q = torch.randn(seqs, heads, 5, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    out = torch.full((seqs, heads, 5, d), 7.0, dtype=dtype, device=DEV)
    count = torch.tensor([5, -3, 100], dtype=torch.int32, device=DEV)  # 5, 0 and 5 tokens
    _attend(shape, pages, q.to(DEV), out, 5, causal=True, count=count)
    torch.cuda.synchronize()
    for s in (0, 2):
        want, tol = P.attend(cache, s, q[s], True, 0, 0, d ** -0.5)
        assert torch.all((out[s].cpu().double() - want).abs() <= tol)
    assert torch.all(out[1] == 7.0)
    # a write whose rows lie in such a page, and rows outside the tensors that hold the tokens
    before = [t.clone() for t in (pages.k.view(torch.uint8), pages.v.view(torch.uint8))]
    pages.lens[:] = torch.tensor([20, 48, 16], dtype=torch.int32)
    x = torch.randn(seqs, heads, 2, d, device=DEV).to(dtype)
    skv.pages_write(shape, pages, x, x, max_new=2)
    first = torch.tensor([-1, 5, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    skv.pages_write(shape, pages, x[0].transpose(0, 1), x[0].transpose(0, 1), first=first,
                    count=torch.tensor([1, 2, 2], dtype=torch.int32, device=DEV), max_new=2)
    o = torch.full((2, heads, d), 7.0, dtype=dtype, device=DEV)
    _attend(shape, pages, x[0].transpose(0, 1), o, 2, first=first,
            count=torch.tensor([1, 2, 2], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(before[0], pages.k.view(torch.uint8)) and torch.equal(before[1], pages.v.view(torch.uint8))
    assert torch.all(o == 7.0)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
def test_strides_and_orders(dtype, cache_dtype):
    # keys and values in one pool, side by side; q, k, v of the tokens in one token-major tensor; output written over q
    d, seqs, heads, kv_heads, page, new = 64, 2, 4, 2, 32, 20
    cache = P.Cache(3, [77, 40], kv_heads, d, page, cache_dtype, dtype)
    both = torch.stack([cache.pool["k"].view(torch.uint8), cache.pool["v"].view(torch.uint8)], 1).to(DEV)
    view = lambda i: both[:, i].view(cache_dtype)
    scales = [None, None] if cache_dtype != E4M3 else list(torch.stack([cache.scales["k"], cache.scales["v"]], 2).to(DEV).unbind(2))
    pages = skv.Pages(view(0), view(1), cache.table.to(DEV), torch.tensor([77, 40], dtype=torch.int32, device=DEV), *scales)
    shape = skv.Shape(seqs, heads, d, dtype)
    fused = torch.randn(seqs, new, heads + 2 * kv_heads, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    on = fused.to(DEV)
    q, k, v = (on[:, :, a:b].transpose(1, 2) for a, b in ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, None)))
    skv.pages_write(shape, pages, k, v)
    _attend(shape, pages, q, q, new, causal=True)
    torch.cuda.synchronize()
    for name, t in (("k", view(0)), ("v", view(1))):
        cache.pool[name] = t.cpu()
        if cache_dtype == E4M3:
            cache.scales[name] = scales[0 if name == "k" else 1].cpu()
    for s in range(seqs):
        for name, a in (("k", heads), ("v", heads + kv_heads)):
            rows = fused[s, :, a:a + kv_heads].transpose(0, 1)
            if cache_dtype == E4M3:
                codes, scale = P.quantised_tensor(rows)
                rows = codes.float().double() * torch.ldexp(torch.ones(()).double(), scale.int() - 127).unsqueeze(-1)
            assert torch.equal(cache.rows(name, s)[:, -new:], rows.double())
        want, tol = P.attend(cache, s, fused[s, :, :heads].transpose(0, 1), True, 0, 0, d ** -0.5)
        assert torch.all((q[s].cpu().double() - want).abs() <= tol)
    assert torch.equal(on[:, :, heads:].cpu(), fused[:, :, heads:])


# Workgroups of many query rows are taken where there are many units: 128 sequences, three of them with rows.
BUSY = (0, 50, 127)


def _check_among_many(seed, heads, kv_heads, d, dtype, cache_dtype, rows, new, **kw):
    print(f"attend among many: {heads}/{kv_heads} heads d {d} {dtype} cache {cache_dtype} rows {rows} new {new} {kw}", flush=True)
    lens, counts = [0] * 128, [0] * 128
    for s, n, t in zip(BUSY, (rows, max(rows - 37, 1), rows), (new, max(new // 2, 1), max(new - 1, 1))):
        lens[s], counts[s] = n, min(n, t)
    _check_lengths(seed, lens, counts, heads, kv_heads, d, dtype, cache_dtype, 16, new, packed=True, **kw)


MASKS = [{}, dict(causal=True), dict(causal=True, window=37, sinks=3), dict(causal=True, window=700, sinks=70)]


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", MASKS)
def test_attend_many_rows_among_many_sequences(dtype, cache_dtype, d, mask):
    for new, rows, group in ((17, 65, 1), (65, 66, 1), (49, 64, 1), (33, 190, 2), (130, 333, 1), (129, 129, 1), (200, 1300, 1)):
        _check_among_many(new, 2 * group, 2, d, dtype, cache_dtype, rows, new, **mask)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_attend_many_rows_over_cut_keys(dtype, cache_dtype, d):
    # (keys are cut in pieces of 16 tiles of 64)
    for new, rows, mask in ((70, 2500, MASKS[1]), (150, 3500, MASKS[0]), (150, 3500, dict(causal=True, window=1900, sinks=5))):
        _check_among_many(rows, 2, 2, d, dtype, cache_dtype, rows, new, **mask)


@pytest.mark.parametrize("dtype,cache_dtype", TYPES)
def test_attend_many_rows_scores_that_rise_and_fall(dtype, cache_dtype):
    for where in (0, 31, 32, 64, 150, 299):
        def change(cache):
            for s in BUSY:
                if where < cache.lens[s]:
                    if cache_dtype == E4M3:
                        at = (int(cache.table[s, where // 16]), 1, where % 16)
                        cache.pool["k"][at], cache.scales["k"][at] = torch.full((128,), 384.0).to(E4M3), 120
                    else:
                        cache.put("k", s, where, 1, torch.full((128,), 3.0))
        for new in (80, 150):
            _check_among_many(where, 2, 2, 128, dtype, cache_dtype, 300, new, scale=2.0, change=change)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window", [0, 5, 40])
def test_many_rows_what_a_token_does_not_see_does_not_reach_it(dtype, d, value, window):
    for new, rows in ((70, 70), (70, 150), (150, 200), (70, 2500), (150, 2500)):
        def change(cache):
            for s in BUSY:
                n = cache.lens[s]
                for r in {0, 3, n - new // 2, n - 1, n - 2, max(0, n - 45)}:
                    if 0 <= r < n:
                        cache.pool["v"][int(cache.table[s, r // 16]), 0, r % 16, 3::7] = value
                cache.pool["k"][int(cache.table[s, (n - 1) // 16]), 1, (n - 1) % 16, 0] = math.nan
                for name in ("k", "v"):
                    cache.pool[name][cache.unused] = math.nan
                    if n % 16:
                        cache.pool[name][int(cache.table[s, n // 16]), :, n % 16:] = math.nan
        _check_among_many(rows, 2, 2, d, dtype, dtype, rows, new, causal=True, window=window, sinks=2, change=change)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", MASKS)
def test_many_rows_codes_and_scales_that_nobody_wrote(dtype, d, mask):
    for new, rows in ((70, 77), (130, 333), (150, 2500)):
        def change(cache):
            for name in ("k", "v"):
                for s in BUSY:
                    n = cache.lens[s]
                    dead = [(p, 0) for p in cache.unused] + ([(int(cache.table[s, n // 16]), n % 16)] if n % 16 else [])
                    for p, slot in dead:
                        cache.pool[name].view(torch.uint8)[p, :, slot:] = 0x7f
                        cache.scales[name][p, :, slot:] = 255
                    for r in (0, 2, n - 30):     # and NaN codes in rows that are seen
                        cache.pool["v"].view(torch.uint8)[int(cache.table[s, r // 16]), 1, r % 16, 1::5] = 0x7f
        _check_among_many(rows, 2, 2, d, dtype, E4M3, rows, new, change=change, **mask)
