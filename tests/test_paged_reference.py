"""The paged-pool operators' plain reference against worked examples, and the
C entry points' refusals, which come before any launch."""
import ctypes

import numpy as np
import pytest

import paged_reference as ref
import paper_2311_00591_amd as coop
from paper_2311_00591_amd.paged import CoopCache, CoopRows


def test_pages_are_placed_given_back_and_refused():
    #       pages 0 1 2 3 4 5 6 7
    kind = [0, 2, 1, 0, 2, 0, 2, 0]
    table = [[1, 4, -1], [6, -1, -1], [-1, -1, -1]]
    # row 0 shrinks to one page (gives back 4), row 1 grows by one, row 2 takes three
    got = ref.page_tables(kind, table, [2, 1, 0], [3, 5, 12], 4)
    assert got[0].tolist() == [[1, -1, -1], [6, 0, -1], [3, 4, 5]]
    assert got[1].tolist() == [1, 2, 3] and got[2].tolist() == [2, 2, 1, 2, 2, 2, 2, 0]
    assert got[3:] == (0, 1)
    # row 0 takes one page, rows 1 and 2 ask for more than is left: row 1 is
    # refused and holds up row 2, which one page would have done
    got = ref.page_tables([0, 2, 0], [[-1, -1], [1, -1], [-1, -1]], [0, 1, 0], [4, 12, 1], 4)
    assert got[3] == 2 and got[1].tolist() == [1, 1, 1]  # 12 tokens: more than two columns
    got = ref.page_tables([0, 2, 0], [[-1] * 3, [1, -1, -1], [-1] * 3], [0, 1, 0], [4, 12, 1], 4)
    assert got[0].tolist() == [[0, -1, -1], [1, -1, -1], [-1, -1, -1]]
    assert got[3:] == (1, 1)


def test_slots_are_the_last_tokens_places():
    table = np.array([[5, 2], [7, -1]])
    got = ref.slot_map(table, [2, 1], [6, 1], [0, 3, 5], 7, 4, 8)
    # sequence 0: positions 3, 4, 5; sequence 1: two new tokens of one; two of none
    assert got.tolist() == [23, 8, 9, -1, 28, -1, -1]
    assert ref.slot_map(table, [1, 1], [6, 1], [0, 3, 5], 5, 4, 7).tolist() == [23, -1, -1, -1, -1]


def test_tree_sight():
    assert ref.seen([-1, 0, 0, 2, -1], 3) == [3, 2, 0]
    assert ref.seen([-1, 0, 0, 2, -1], 4) == [4]
    assert ref.seen([-1, 1, 1, 0], 1) is None   # its own parent
    assert ref.seen([-1, 1, 1, 0], 2) == [2]    # its parent is void
    assert ref.seen(None, 2) == [0, 1, 2]


def test_e4m3_numbers():
    v = ref.e4m3_values()
    assert len(v) == 253 and v.max() == 448 and v[v > 0].min() == 2.0**-9


NZ = 64  # non-null, 16-byte aligned, never dereferenced


def _lib():
    return coop.load_library()


def test_page_tables_refusals():
    def call(pages=8, rows=2, cols=4, page=16, taken=2, wsb=1 << 20, **ptr):
        a = dict(kind=0x1000000, table=0x2000000, held=0x3000000, lengths=0x4000000,
                 table_out=0x5000000, held_out=0x6000000, kind_out=0x7000000, status=0x8000000, free=0x9000000, ws=0xa000000)
        a.update(ptr)
        return _lib().coop_page_tables(a["kind"], pages, a["table"], rows, cols, a["held"],
                                       a["lengths"], page, taken, a["table_out"], a["held_out"],
                                       a["kind_out"], a["status"], a["free"], a["ws"], wsb, None)

    for name in ("kind", "table", "held", "lengths", "table_out", "held_out", "kind_out", "status",
                 "free"):
        assert call(**{name: None}) == -1, name
    # (a pool of up to 2^17 pages and 2^9 rows needs no workspace)
    for large in (dict(pages=1 << 20), dict(rows=513)):
        assert call(ws=None, **large) == -2 and call(wsb=8, **large) == -2
        assert call(ws=0xa000008, **large) == -1
    assert call(page=0) == -1 and call(taken=0) == -1 and call(taken=3) == -1
    for big in ("pages", "rows", "cols"):
        assert call(**{big: 1 << 31}) == -1, big
    # an output may be its own input, not another one or a part of one
    assert call(table_out=0x2000004) == -1
    assert call(table_out=0x3000000) == -1
    assert call(kind_out=0x4000000) == -1
    out = ctypes.c_size_t()
    assert _lib().coop_page_tables_workspace_size(1, 1, None) == -1
    assert _lib().coop_page_tables_workspace_size(1 << 31, 1, ctypes.byref(out)) == -1
    assert coop.page_tables_workspace_size(100000, 64) == 0
    assert 0 < coop.page_tables_workspace_size(1 << 20, 64) < 1 << 16


def test_slot_map_refusals():
    def call(rows=2, cols=4, tokens=3, page=16, pages=8, **ptr):
        a = dict(table=NZ, held=NZ, lengths=NZ, off=NZ, out=NZ)
        a.update(ptr)
        return _lib().coop_slot_map(a["table"], rows, cols, a["held"], a["lengths"], a["off"],
                                    tokens, page, pages, a["out"], None)

    assert call(tokens=0, out=None) == 0
    for name in ("table", "held", "lengths", "off", "out"):
        assert call(**{name: None}) == -1, name
    assert call(page=0) == -1 and call(rows=1 << 31) == -1 and call(tokens=1 << 61) == -1


def _cache_of(**kw):
    d = dict(k=NZ, v=NZ, k_stride=(2048, 128, 64), v_stride=(2048, 128, 64), k_scale=None,
             v_scale=None, num_pages=4, page_size=16, heads=2, dim=64, type=0)
    d.update(kw)
    return CoopCache(d["k"], d["v"], d["k_stride"], d["v_stride"], d["k_scale"], d["v_scale"],
                     d["num_pages"], d["page_size"], d["heads"], d["dim"], d["type"])


BAD_CACHES = [dict(k=None), dict(v=None), dict(k=NZ + 8), dict(v=NZ + 2),
              dict(k_stride=(2048, 132, 64)), dict(v_stride=(2047, 128, 64)), dict(dim=0),
              dict(dim=60), dict(dim=264), dict(heads=0), dict(heads=1 << 17), dict(page_size=0),
              dict(num_pages=1 << 31), dict(page_size=1 << 31), dict(type=1), dict(type=3),
              dict(type=2), dict(type=2, k_scale=NZ), dict(k_scale=NZ, v_scale=NZ),
              dict(type=2, k_scale=NZ, v_scale=NZ, dim=72),
              dict(type=2, k_scale=NZ, v_scale=NZ, k_stride=(2048, 128, 72)),
              dict(k_stride=(1 << 41, 128, 64))]
ROWS = (128, 64)
BAD_ROWS = [(None, ROWS), (NZ + 8, ROWS), (NZ, (128, 60)), (NZ, (12, 64)), (NZ, (1 << 41, 64))]


def test_cache_write_refusals():
    def call(k=(NZ, ROWS), v=(NZ, ROWS), type=0, slots=NZ, tokens=3, cache={}):
        return _lib().coop_cache_write(CoopRows(*k), CoopRows(*v), type, slots, tokens,
                                       _cache_of(**cache), None)

    assert call(tokens=0) == 0 and call(cache=dict(num_pages=0), k=(None, ROWS)) == 0
    for bad in BAD_CACHES:
        assert call(cache=bad) == -1, bad
    for bad in BAD_ROWS:
        assert call(k=bad) == -1 and call(v=bad) == -1, bad
    assert call(type=2) == -1 and call(slots=None) == -1 and call(tokens=1 << 41) == -1
    assert _lib().coop_cache_write(None, None, 0, NZ, 3, None, None) == -1


def test_tree_attention_refusals():
    def call(q=(NZ, ROWS), k=(NZ, ROWS), v=(NZ, ROWS), type=0, q_heads=4, tokens=3, off=NZ,
             parents=NZ, table=NZ, cols=4, lengths=NZ, requests=2, out=NZ, ws=NZ, wsb=1 << 30,
             cache={}):
        return _lib().coop_tree_attention(CoopRows(*q), CoopRows(*k), CoopRows(*v), type, q_heads,
                                          tokens, off, parents, _cache_of(**cache), table, cols,
                                          lengths, requests, 0.125, out, ws, wsb, None)

    assert call(tokens=0, out=None) == 0 and call(requests=0) == 0
    for bad in BAD_CACHES:
        assert call(cache=bad) == -1, bad
    for bad in BAD_ROWS:
        assert call(q=bad) == -1 and call(k=bad) == -1 and call(v=bad) == -1, bad
    assert call(type=2) == -1
    for name in ("off", "table", "lengths", "out"):
        assert call(**{name: None}) == -1, name
    assert call(out=NZ + 8) == -1 and call(ws=NZ + 8) == -1
    assert call(ws=None) == -2 and call(wsb=4096) == -2
    assert call(q_heads=5) == -1 and call(q_heads=0) == -1
    assert call(tokens=1 << 30) == -1 and call(requests=1 << 31) == -1 and call(cols=1 << 31) == -1
    assert _lib().coop_tree_attention(None, None, None, 0, 4, 3, NZ, None, None, NZ, 4, NZ, 2, 1.0,
                                      NZ, NZ, 1 << 30, None) == -1
    out = ctypes.c_size_t()
    size = _lib().coop_tree_attention_workspace_size
    assert size(2, 3, 4, 2, 64, None) == -1
    for bad in ((2, 3, 5, 2, 64), (2, 3, 4, 0, 64), (2, 3, 4, 2, 260), (2, 1 << 31, 4, 2, 64)):
        assert size(*bad, ctypes.byref(out)) == -1, bad


def test_no_cpu_fallback():
    import torch
    i32, i64 = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    pool = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        coop.page_tables(torch.zeros(4, dtype=torch.uint8), i32, i32[0], i64[:1], 16)
    with pytest.raises(ValueError, match="GPU"):
        coop.slot_map(i32, i32[0], i64[:1], i64, 1, 16, 4)
    with pytest.raises(ValueError, match="GPU"):
        coop.cache_write(x, x, i64[:1], pool, pool)
    with pytest.raises(ValueError, match="GPU"):
        coop.tree_attention(x, x, x, pool, pool, i32, i64[:1], i64)
