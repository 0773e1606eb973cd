"""Host-only checks of the paged cache's entry points: what they refuse (pointers below are fake but aligned and never
dereferenced: every call is refused before a launch), the host check of tables, and the 64-bit definitions that the GPU
tests compare with.  No GPU needed."""
import ctypes
import itertools
import math
import os
import random

import numpy as np
import pytest
import torch

import paper_2505_19602_amd as skv
import pages_util as P
from paper_2505_19602_amd import binding as B
from paper_2505_19602_amd import build as hip_build

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(skv.lib_path()):
        hip_build.build(force=True)
    return skv.lib()


def _err(L):
    return L.scalekv_last_error().decode()


def _shape(**kw):
    base = dict(n_seq=2, n_head=4, head_dim=128, dtype=BF16, sm_scale=0.0)
    base.update(kw)
    return B._CShape(*base.values())


def _pages(**kw):
    """Ten pages of 32 rows, two KV heads, of 128 elements: 16 KB a page in 16 bits."""
    d, heads, rows = 128, 2, 32
    base = dict(k=0x1000000, v=0x2000000, k_scale=0x3000000, v_scale=0x3100000, page_stride=heads * rows * d,
                head_stride=rows * d, scale_page_stride=heads * rows, scale_head_stride=rows, n_page=10, n_kv_head=heads,
                page_rows=rows, dtype=BF16, table=0x4000000, table_width=5, len=0x4100000)
    base.update(kw)
    return B._CPages(*base.values())


def _rows(**kw):
    base = dict(ptr=0x5000000, seq_stride=4 * 8 * 128, head_stride=8 * 128, row_stride=128, n_row=8)
    base.update(kw)
    return B._CRows(*base.values())


def _chunk(**kw):
    base = dict(max_new=8, first=0, count=0)
    base.update(kw)
    return B._CChunk(*base.values())


def _mask(causal=1, window=0, n_sink=0):
    return B._CMask(causal, window, n_sink)


def _ref(x):
    return None if x is None else ctypes.byref(x)


BAD_SHAPES = [(dict(n_seq=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=E4M3), UNSUPPORTED),
              (dict(n_seq=70000), UNSUPPORTED), (dict(sm_scale=math.nan), INVALID)]
BAD_SIZES = [(dict(dtype=7), UNSUPPORTED, "dtype"), (dict(dtype=F32), UNSUPPORTED, "neither the shape's"),
             (dict(page_rows=24), UNSUPPORTED, "power of two"), (dict(page_rows=8), UNSUPPORTED, "page_rows"),
             (dict(page_rows=512), UNSUPPORTED, "page_rows"), (dict(page_rows=0), UNSUPPORTED, "page_rows"),
             (dict(page_rows=-32), UNSUPPORTED, "page_rows"), (dict(n_page=0), INVALID, "n_page"),
             (dict(n_kv_head=3), INVALID, "divide"), (dict(n_kv_head=0), INVALID, "n_kv_head"),
             (dict(n_kv_head=8), INVALID, "divide"), (dict(table_width=0), INVALID, "table_width"),
             (dict(table_width=1 << 26), UNSUPPORTED, "2^30")]
BAD_PAGES = BAD_SIZES + [
    (dict(k=0), INVALID, "pages.k"), (dict(v=0), INVALID, "pages.v"), (dict(k=0x1000008), INVALID, "aligned"),
    (dict(head_stride=32 * 128 - 8), INVALID, "head_stride"), (dict(head_stride=32 * 128 + 4), INVALID, "multiple"),
    (dict(page_stride=2 * 32 * 128 - 8), INVALID, "page_stride"), (dict(page_stride=1 << 41), INVALID, "page_stride"),
    (dict(page_stride=1 << 40, n_page=1 << 20), UNSUPPORTED, "too far"),
    (dict(dtype=E4M3, k_scale=0), INVALID, "scale"), (dict(dtype=E4M3, scale_head_stride=31), INVALID, "scale_head_stride"),
    (dict(dtype=E4M3, scale_page_stride=63), INVALID, "scale_page_stride"),
    (dict(table=0), INVALID, "table"), (dict(len=0), INVALID, "len")]
BAD_CHUNKS = [(dict(max_new=0), INVALID, "max_new"), (dict(max_new=-1), INVALID, "max_new"),
              (dict(max_new=9), INVALID, "n_row"), (dict(max_new=1 << 27), UNSUPPORTED, "too large")]
BAD_ROWS = [(dict(ptr=0), INVALID, "ptr"), (dict(ptr=0x5000004), INVALID, "aligned"), (dict(row_stride=-128), INVALID, "stride"),
            (dict(head_stride=100), INVALID, "stride"), (dict(seq_stride=1 << 41), INVALID, "stride"),
            (dict(n_row=-1), INVALID, "n_row"), (dict(n_row=7), INVALID, "n_row"),
            (dict(n_row=2 ** 31 - 1, row_stride=1 << 39), UNSUPPORTED, "too far")]


def _write(L, shape=None, pages=None, k=None, v=None, chunk=None):
    return L.scalekv_pages_write(_ref(shape or _shape()), _ref(pages or _pages()), _ref(k or _rows()),
                                 _ref(v or _rows(ptr=0x6000000)), _ref(chunk or _chunk()), None)


def _read(L, shape=None, pages=None, n_row=8, k=None, v=None):
    kv = lambda at: B._CKv(at, 4 * 10 * 128, 10 * 128, 10)
    return L.scalekv_pages_read(_ref(shape or _shape()), _ref(pages or _pages()), None, n_row, _ref(k or kv(0x5000000)),
                                _ref(v or kv(0x6000000)), None)


def _attend(L, shape=None, pages=None, q=None, chunk=None, mask=None, out=None, ws=None, ws_bytes=0):
    return L.scalekv_pages_attend(_ref(shape or _shape()), _ref(pages or _pages()), _ref(q or _rows()),
                                  _ref(chunk or _chunk()), _ref(mask or _mask()), _ref(out or _rows(ptr=0x6000000)),
                                  ctypes.c_void_p(ws), ctypes.c_size_t(ws_bytes), None)


def _need(L, shape=None, pages=None, max_new=8, mask=None):
    out = ctypes.c_size_t(77)
    st = L.scalekv_pages_workspace_bytes(_ref(shape or _shape()), _ref(pages or _pages()), max_new, _ref(mask or _mask()),
                                         ctypes.byref(out))
    return st, out.value


def test_shapes_pages_and_chunks_that_are_refused(L):
    for kw, status in BAD_SHAPES:
        s = _shape(**kw)
        assert _write(L, s) == _read(L, s) == _attend(L, s) == _need(L, s)[0] == status, kw
    for kw, status, word in BAD_PAGES:
        for call in (_write, _read, _attend):
            assert call(L, pages=_pages(**kw)) == status, (call, kw)
            assert word in _err(L), (kw, _err(L))
    for kw, status, word in BAD_SIZES:
        assert _need(L, pages=_pages(**kw))[0] == status and word in _err(L), kw
    for kw, status, word in BAD_CHUNKS:
        for call in (_write, _attend):
            assert call(L, chunk=_chunk(**kw)) == status and word in _err(L), (call, kw, _err(L))
    for kw, status, word in BAD_ROWS:
        bad = _rows(**kw)
        for got in (_write(L, k=bad), _write(L, v=bad), _attend(L, q=bad), _attend(L, out=bad)):
            assert got == status and word in _err(L), (kw, _err(L))
    for f, n in ((L.scalekv_pages_write, 6), (L.scalekv_pages_read, 7), (L.scalekv_pages_attend, 9)):
        assert f(None, *([None] * (n - 1))) == INVALID
        assert f(ctypes.byref(_shape()), *([None] * (n - 1))) == INVALID and "pages is NULL" in _err(L)
    assert L.scalekv_pages_workspace_bytes(ctypes.byref(_shape()), ctypes.byref(_pages()), 1, None, None) == INVALID
    assert _need(L, max_new=0)[0] == INVALID


def test_masks_workspaces_and_overlaps_that_are_refused(L):
    for mask, word in ((_mask(causal=2), "causal"), (_mask(window=-1), "window"), (_mask(n_sink=-1), "n_sink")):
        assert _attend(L, mask=mask) == INVALID and word in _err(L)
        assert _need(L, mask=mask)[0] == INVALID
    # a single token of two sequences over a long table needs a workspace
    long, one = _pages(table_width=4000), _chunk(max_new=1)
    st, need = _need(L, pages=long, max_new=1)
    assert st == OK and need > 0
    assert _attend(L, pages=long, chunk=one) == WORKSPACE and "needed" in _err(L)
    assert _attend(L, pages=long, chunk=one, ws=0x7000000, ws_bytes=need - 1) == WORKSPACE
    assert _attend(L, pages=long, chunk=one, ws=0x7000008, ws_bytes=need) == INVALID and "aligned" in _err(L)
    for at in (0x1000000, 0x2000000, 0x5000000, 0x6000000):
        assert _attend(L, pages=long, chunk=one, ws=at, ws_bytes=need) == INVALID and "workspace overlaps" in _err(L)
    # rows of out that coincide, out on q but not exactly, out and new rows in the pool
    for kw in (dict(head_stride=0), dict(row_stride=0), dict(seq_stride=0)):
        assert _attend(L, out=_rows(ptr=0x6000000, **kw)) == INVALID and "coincide" in _err(L)
    assert _attend(L, out=_rows(ptr=0x5000000 + 256)) == INVALID and "overlaps q" in _err(L)
    assert _attend(L, out=_rows(row_stride=256)) == INVALID and "overlaps q" in _err(L)
    for at in (0x1000000, 0x2000000 + 9 * 16384):
        assert _attend(L, out=_rows(ptr=at)) == INVALID and "overlaps the pool" in _err(L)
        assert _write(L, k=_rows(ptr=at)) == _write(L, v=_rows(ptr=at)) == INVALID and "overlaps the pool" in _err(L)
        assert _read(L, k=B._CKv(at, 4 * 1280, 1280, 10)) == INVALID and "overlaps the pool" in _err(L)
    q8 = _pages(dtype=E4M3)
    assert _attend(L, pages=q8, out=_rows(ptr=0x3000000)) == INVALID
    assert _read(L, v=B._CKv(0x5000000, 4 * 1280, 1280, 10)) == INVALID and "overlap" in _err(L)
    assert _read(L, n_row=11) == INVALID and "capacity" in _err(L)
    assert _read(L, n_row=-1) == INVALID
    assert _read(L, n_row=0) == OK                                   # nothing to do needs no device


def test_keys_and_values_that_share_bytes_are_refused(L):
    # keys and values page by page in turn are fine, a few bytes off they are not (no call here gets as far as a launch)
    bytes_of_page = 2 * 32 * 128 * 2
    for gap in (0, 256, -256, 32 * 128 * 2 - 16, bytes_of_page, -bytes_of_page, 9 * bytes_of_page, 32 * 128 * 2,
                -32 * 128 * 2, 10 * bytes_of_page - 16):
        assert _write(L, pages=_pages(v=0x1000000 + gap)) == INVALID, gap
        assert "pages.k and pages.v overlap" in _err(L)
    apart = 2 * bytes_of_page // 2                                    # k pages, v pages in turn
    for gap in (16, 32 * 128 * 2 - 16, -16):
        assert _write(L, pages=_pages(page_stride=2 * 2 * 32 * 128, v=0x1000000 + gap)) == INVALID
    assert _write(L, pages=_pages(page_stride=2 * 2 * 32 * 128, v=0x1000000 + apart + 16)) == INVALID
    assert _write(L, pages=_pages(dtype=E4M3, v_scale=0x3000000 + 40)) == INVALID and "v_scale overlap" in _err(L)
    assert _write(L, pages=_pages(dtype=E4M3, k_scale=0x1000000)) == INVALID and "scales overlap" in _err(L)


def test_the_workspace_covers_every_size_and_is_not_asked_for_where_rows_abound(L):
    # sums of every workgroup that there may be: no more than keys can be cut for, and than there are tiles of 128 keys
    for n_seq, heads, kv, width, new in ((1, 8, 1, 4096, 1), (2, 32, 8, 4096, 1), (1, 1, 1, 1, 1), (64, 32, 8, 125, 1)):
        st, need = _need(L, _shape(n_seq=n_seq, n_head=heads), _pages(n_kv_head=kv, table_width=width), new)
        units, parts = n_seq * kv, -(-width * 32 // 128)
        assert st == OK and need % 4 == 0 and need <= min(512 + units, units * parts) * heads // kv * 130 * 4 + 8 * n_seq
    assert _need(L, _shape(n_seq=16, n_head=16), _pages(n_kv_head=16, table_width=200), 4096) == (OK, 0)


def _check(L, table, lens, count=None, first=None, max_new=None, n_row=0, **kw):
    width = len(table[0])
    ints = lambda x: None if x is None else (ctypes.c_int32 * len(x))(*x)
    chunk = None if max_new is None else ctypes.byref(_chunk(max_new=max_new))
    return L.scalekv_pages_check(ctypes.byref(_shape(n_seq=len(table))), ctypes.byref(_pages(table_width=width, **kw)),
                                 ints([x for r in table for x in r]), ints(lens), chunk, ints(first), ints(count), n_row)


def test_packed_tensors_without_rows_are_fine(L):
    none, chunk = _rows(ptr=0, n_row=0, seq_stride=0), _chunk(first=0x7000000, count=0x7100000)
    assert _write(L, k=none, v=none, chunk=chunk) == OK and _attend(L, q=none, out=none, chunk=chunk) == OK
    assert _write(L, k=none, v=none) == INVALID                       # (not packed: max_new rows are needed)


def test_tables_with_mistakes_are_named(L):
    good = [[0, 1, -1], [2, 9, 5]]
    assert _check(L, good, [40, 96]) == OK                           # (entries behind the last page are not used)
    assert _check(L, good, [40, 96], count=[8, 0], max_new=8, n_row=8) == OK
    assert _check(L, good, [0, 0]) == OK
    for table, lens, kw, word in (
            (good, [65, 96], {}, "table[0][2]"), ([[0, 10, 1], [2, 3, 4]], [40, 40], {}, "table[0][1] = 10"),
            ([[0, -7, 1], [2, 3, 4]], [40, 40], {}, "table[0][1] = -7"), (good, [-1, 5], {}, "len[0]"),
            (good, [40, 97], {}, "len[1]"), (good, [40, 96], dict(max_new=8, count=[9, 0], n_row=8), "count[0]"),
            (good, [40, 96], dict(max_new=8, count=[-1, 0], n_row=8), "count[0]"),
            (good, [40, 3], dict(max_new=8, n_row=8), "count[1]"), (good, [40, 96], dict(max_new=8, n_row=7), "sequence 0"),
            (good, [40, 96], dict(max_new=8, first=[0, 5], n_row=8), "sequence 1"),
            (good, [40, 96], dict(max_new=8, first=[-1, 0], n_row=8), "sequence 0")):
        assert _check(L, table, lens, **kw) == INVALID and word in _err(L), (kw, _err(L))
    # a shared prefix is fine until somebody writes to it
    shared = [[0, 1, 2], [0, 1, 3]]
    assert _check(L, shared, [70, 80]) == OK
    assert _check(L, shared, [70, 80], count=[6, 16], max_new=16, n_row=16) == OK
    assert _check(L, shared, [70, 80], count=[7, 16], max_new=16, n_row=16) == INVALID and "page 1" in _err(L)
    assert _check(L, [[0, 1, 0], [2, 3, 4]], [70, 80], count=[1, 0], max_new=1, n_row=1) == INVALID and "page 0" in _err(L)
    assert L.scalekv_pages_check(ctypes.byref(_shape()), ctypes.byref(_pages()), None, None, None, None, None, 0) == INVALID


def test_the_binding_refuses_tensors_that_are_not_what_it_says():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for args in ((k.half(), k.half(), table, lens), (k, k.float(), table, lens), (k, k[:2], table, lens), (k, k, table, lens)):
        with pytest.raises(skv.ScaleKVError):                         # (the last: not on a device)
            skv.Pages(*args)


def test_packed_tensors_of_different_lengths_are_refused(L):
    # a sequence's tokens lie at the same rows of both: behind the end of the shorter one they would be left out, unsaid
    chunk = _chunk(first=0x7000000, count=0x7100000)
    rows = lambda n, at=0x5000000: _rows(ptr=at if n else 0, seq_stride=0, n_row=n)
    for a, b in ((8, 5), (5, 8), (8, 0), (0, 8), (1, 2)):
        assert _write(L, k=rows(a), v=rows(b, 0x6000000), chunk=chunk) == INVALID, (a, b)
        assert f"k_new has {a} rows and v_new {b}" in _err(L)
        assert _attend(L, q=rows(a), out=rows(b, 0x6000000), chunk=chunk) == INVALID, (a, b)
        assert f"q has {a} rows and out {b}" in _err(L)
    # rows of a sequence that lie behind max_new are not looked at: dense tensors may have more of them
    inside = 0x2000000                                                # (refused behind that check, before a launch)
    assert _attend(L, q=_rows(n_row=9), out=_rows(ptr=inside)) == INVALID and "overlaps the pool" in _err(L)
    assert _write(L, k=_rows(n_row=9), v=_rows(ptr=inside)) == INVALID and "overlaps the pool" in _err(L)


def test_packed_rows_that_two_sequences_share_are_named(L):
    def check(first, count, max_new=8, n_row=30):
        ints = lambda x: None if x is None else (ctypes.c_int32 * len(x))(*x)
        return L.scalekv_pages_check_packed(ctypes.byref(_shape(n_seq=len(first), n_head=1)),
                                            ctypes.byref(_chunk(max_new=max_new)), ints(first), ints(count), n_row)
    for first, count in (([0, 8], None), ([8, 0], None), ([0, 3, 5], [3, 2, 8]), ([5, 0, 3], [8, 3, 2]), ([22, 0], [8, 8]),
                         ([4, 4, 4], [0, 5, 0]), ([0, -9, 99], [8, 0, 0]), ([0, 5, 3], [5, 8, 0])):
        assert check(first, count) == OK, (first, count, _err(L))
    for first, count, word in (([0, 7], None, "sequences 0 and 1"), ([3, 0, 5], [3, 2, 8], "sequences 0 and 2"),
                               ([4, 4], [1, 1], "sequences 0 and 1"), ([0, 20, 2], [8, 1, 1], "sequences 0 and 2"),
                               ([0, 2, 20], [8, 1, 1], "sequences 0 and 1"), ([0, 23], None, "rows 23..30 of sequence 1"),
                               ([0, -1], [8, 1], "sequence 1"), ([0, 8], [8, 9], "count[1]"), ([0, 8], [-1, 8], "count[0]"),
                               ([0, 2 ** 31 - 1], [1, 8], "sequence 1")):
        assert check(first, count) == INVALID and word in _err(L), (first, count, _err(L))
    assert check([0, 0], None, max_new=0) == INVALID and "max_new" in _err(L)
    one = _shape()
    assert L.scalekv_pages_check_packed(ctypes.byref(one), ctypes.byref(_chunk()), None, None, 8) == INVALID
    assert "first is NULL" in _err(L)
    assert L.scalekv_pages_check_packed(ctypes.byref(one), None, None, None, 8) == INVALID and "chunk is NULL" in _err(L)
    assert L.scalekv_pages_check_packed(None, None, None, None, 8) == INVALID


def test_the_binding_checks_packed_rows_where_it_is_told_to():
    class Sizes:                                                      # (pages without a device: sizes alone are looked at)
        table, c = torch.zeros(2, 3, dtype=torch.int32), _pages(table_width=3)
    shape, table = skv.Shape(2, 4, 128, torch.bfloat16), [[0, 1, 2], [3, 4, 5]]
    call = lambda first, **kw: skv.pages_check(shape, Sizes, table, [40, 90], first=first, max_new=4, n_row=8, **kw)
    call([4, 0], packed=True)
    call([0, 3])                                                      # a padded batch: its rows are those of each sequence
    with pytest.raises(skv.ScaleKVError, match="sequences 0 and 1"):
        call([0, 3], packed=True)
    for kw in (dict(first=None, max_new=4), dict(first=[0, 4])):
        with pytest.raises(skv.ScaleKVError, match="packed"):
            skv.pages_check(shape, Sizes, table, [40, 90], n_row=8, packed=True, **kw)


def test_rows_of_out_that_coincide_are_refused_whatever_the_strides(L):
    # every stride holds a row, and yet two rows share bytes; the calls that pass come to the check against the pool, and end there
    d = 128

    def verdict(seqs, heads, rows, seq, head, row, n_row=0, **more):
        out = _rows(ptr=0x1000000, seq_stride=seq, head_stride=head, row_stride=row, n_row=n_row or rows)
        q = _rows(ptr=0x40000000, n_row=n_row or rows)
        st = _attend(L, _shape(n_seq=seqs, n_head=heads), q=q, out=out, chunk=_chunk(max_new=rows, **more))
        assert st == INVALID and ("coincide" in _err(L)) != ("overlaps the pool" in _err(L)), (st, _err(L))
        return "coincide" in _err(L)

    assert verdict(1, 4, 8, 0, d, d) and verdict(1, 4, 8, 0, 7 * d, d) and verdict(1, 4, 8, 0, d, 3 * d)
    assert verdict(2, 4, 8, 8 * d, 8 * d, d) and verdict(2, 2, 1, d, d, 0) and verdict(2, 2, 8, 8 * d, 16 * d, d + 8)
    assert not verdict(1, 4, 8, 0, d, 4 * d) and not verdict(1, 4, 8, 0, 8 * d, d) and not verdict(2, 2, 1, d, 2 * d, 0)
    assert not verdict(1, 2, 4, 0, 3 * d, 2 * d)                      # (no dimension holds another whole: rows 0 2 4 6, 3 5 7 9)
    assert verdict(1, 4, 4, 0, 3 * d, 2 * d)
    assert not verdict(2, 4, 4, 4 * d, 8 * d, d, n_row=8)             # (rows behind max_new are not written)
    assert verdict(2, 4, 4, 4 * d, 8 * d, d, n_row=8, first=0x7000000)   # (but where first places the tokens they may be)
    assert not verdict(2, 4, 4, 0, d, 4 * d, n_row=8, first=0x7000000)   # packed
    rng = random.Random(1)
    found = [0, 0]
    for _ in range(3000):
        n = [rng.choice((1, 2, 2, 4, 6)), rng.choice((2, 4, 6)), rng.randint(1, 5)]
        strides = [d + 8 * rng.randint(0, rng.choice((3, 40, 120))) for _ in range(3)]
        starts = sorted(sum(x * y for x, y in zip(at, strides)) for at in itertools.product(*map(range, n)))
        want = any(b - a < d for a, b in zip(starts, starts[1:]))
        assert verdict(*n, *strides) == want, (n, strides)
        found[want] += 1
    assert min(found) > 100
    # many rows, in dimensions that lie in each other
    assert not verdict(1024, 2, 8, 8 * 8 * d, 8 * d, d) and verdict(1024, 2, 8, 2 * 8 * d, 8 * d - 8, d)


def test_scales_may_lie_beside_the_codes_of_their_page(L):
    # packed tensors without rows: an accepted call ends before a launch
    none, chunk = _rows(ptr=0, n_row=0, seq_stride=0), _chunk(first=0x7000000, count=0x7100000)

    def verdict(at, page, head, scale_head, n_page=10, scale_page=None, heads=2):
        pages = _pages(dtype=E4M3, v=0x9000000, page_stride=page, head_stride=head, n_page=n_page, n_kv_head=heads,
                       scale_page_stride=scale_page or page, scale_head_stride=scale_head, k_scale=0x1000000 + at,
                       v_scale=0xa000000)
        st = _write(L, _shape(n_head=heads), pages, none, none, chunk)
        assert st == OK or (st == INVALID and "scales overlap the pool" in _err(L)), (st, _err(L))
        return st == OK

    unit = 32 * 128                                                   # codes of a head: 4096 bytes, scales: 32
    record = 2 * (2 * unit + 64)
    assert verdict(2 * unit, record, unit, 32) and verdict(2 * unit + 64, record, unit, 32)
    assert verdict(unit, record, unit + 32, unit + 32)                # head by head: codes, scales
    assert verdict(-64, record, unit, 32) and verdict(2 * unit - record, record, unit, 32)
    assert not verdict(2 * unit - 1, record, unit, 32) and not verdict(record - 63, record, unit, 32)
    assert not verdict(unit - 1, record, unit + 32, unit + 32) and not verdict(unit + 1, record, unit + 32, unit + 32)
    assert not verdict(2 * unit, record, unit, 32, scale_page=record + 16)   # pages' strides that differ: refused within the span
    assert verdict(10 * record, record, unit, 32) and not verdict(10 * record, record, unit, 32, n_page=11, scale_page=64)
    # keys and values with their scales in one record
    pages = _pages(dtype=E4M3, v=0x1000000 + 2 * unit, page_stride=2 * 2 * unit + 128, k_scale=0x1000000 + 4 * unit,
                   v_scale=0x1000000 + 4 * unit + 64, scale_page_stride=2 * 2 * unit + 128)
    assert _write(L, pages=pages, k=none, v=none, chunk=chunk) == OK
    rng, found = random.Random(2), [0, 0]
    for _ in range(3000):
        heads, n_page = rng.choice((1, 2, 4)), rng.randint(1, 4)
        head, scale_head = unit + 16 * rng.randint(0, 9), rng.choice((32, 40, unit, unit + 16 * rng.randint(0, 9)))
        page = max(heads * head, heads * scale_head) + 16 * rng.randint(0, 30)
        if rng.random() < 0.5:                                        # around a head's or a page's end
            at = rng.randint(-n_page, n_page) * page + rng.randint(0, heads) * head + rng.randint(-40, 200)
        else:
            at = rng.randint(-n_page * page - 9, n_page * page + 9)
        codes = [(i * page + h * head, i * page + h * head + unit) for i in range(n_page) for h in range(heads)]
        scales = [(at + i * page + h * scale_head, at + i * page + h * scale_head + 32) for i in range(n_page) for h in range(heads)]
        want = not any(a < y and x < b for a, b in codes for x, y in scales)
        assert verdict(at, page, head, scale_head, n_page, heads=heads) == want, (at, page, head, scale_head, n_page, heads)
        found[want] += 1
    assert min(found) > 300, found


def test_as_many_token_rows_as_the_kernels_can_count(L):
    # rows of a unit are counted in int32, in row groups of up to 128: the last group's end has to fit
    d, heads = 64, 64
    pages = _pages(n_kv_head=1, head_stride=32 * d, page_stride=32 * d)
    for new, status in (((2 ** 31 - 256) // heads, OK), ((2 ** 31 - 256) // heads + 1, UNSUPPORTED),
                        ((2 ** 31 - 1) // d, UNSUPPORTED)):
        st, need = _need(L, _shape(n_seq=1, n_head=heads, head_dim=d), pages, new)
        assert st == status and (st != OK or need == 0) and (st == OK or "too large" in _err(L)), (new, st, need)


# ---- the definitions in 64 bits that the GPU tests use

def test_codes_are_the_nearest_e4m3_values_ties_to_even():
    values = sorted({float(v) for v in torch.arange(256, dtype=torch.uint8).view(P.E4M3).float() if math.isfinite(v)})
    assert len(values) == 253 and values[-1] == 448.0 and min(v for v in values if v > 0) == 2.0 ** -9
    even = {float(v) for v in torch.arange(0, 256, 2, dtype=torch.uint8).view(P.E4M3).float()}
    for a, b in zip(values, values[1:]):
        for x, want in ((a, a), (a + 0.25 * (b - a), a), (a + 0.75 * (b - a), b), ((a + b) / 2, a if a in even else b)):
            assert P.nearest_code(x) == want
    x = torch.randn(50, 64, generator=torch.Generator().manual_seed(1)) * 2.0 ** torch.randint(-40, 40, (50, 1)).float()
    x[3] = 0
    x[4, 7], x[5, 8] = math.inf, math.nan
    codes, scale = P.quantised_tensor(x)
    for i in range(50):
        row, k = P.quantised(x[i].double().numpy())
        assert int(scale[i]) == k + 127 and np.array_equal(codes[i].float().numpy(), row, equal_nan=True)
        fine = torch.isfinite(x[i])
        err = (x[i].double().numpy() - np.ldexp(row, k))[fine]
        assert np.all(np.abs(err) <= np.maximum(2.0 ** -4 * np.abs(x[i].double().numpy()[fine]), 2.0 ** (k - 10)))


def test_the_64_bit_attention_is_a_softmax_over_what_a_token_sees():
    cache = P.Cache(1, [50], 1, 64, 16, torch.float32, torch.float32)
    q = torch.randn(2, 9, 64, generator=torch.Generator().manual_seed(3))
    k, v = cache.rows("k", 0)[0], cache.rows("v", 0)[0]
    for causal, window, sinks in ((False, 0, 0), (True, 0, 0), (True, 5, 2), (False, 5, 0)):
        hidden = torch.stack([~P.sees(41 + t, 50, causal, window, sinks) for t in range(9)])
        want = torch.softmax((q.double() @ k.t() / 8).masked_fill(hidden, -math.inf), -1) @ v
        out, tol = P.attend(cache, 0, q, causal, window, sinks, 0.125)
        assert torch.allclose(out, want, atol=1e-12) and torch.all(tol > 0) and float(tol.max()) < 1e-2
    assert P.sees(0, 4, True, 1, 0).tolist() == [True, False, False, False]
    assert P.sees(3, 5, True, 2, 1).tolist() == [True, False, True, True, False]
    assert not P.sees(-2, 5, True, 0, 3).any()
