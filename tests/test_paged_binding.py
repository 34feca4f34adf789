"""The paged pools' binding and C refusals that need no GPU."""
import subprocess
import sys

import pytest

import paper_2311_00591_amd as coop
from conftest import ROOT
from paper_2311_00591_amd.paged import CoopCache, CoopRows


def test_the_package_imports_where_torch_has_no_gpu_support():
    """A torch built without GPU support lacks some names of torch._C; the
    package imports there, as it did without the paged pools."""
    code = ("import torch\n"
            "for name in [n for n in dir(torch._C) if n.startswith('_cuda_')]:\n"
            "    delattr(torch._C, name)\n"
            "import paper_2311_00591_amd as coop\n"
            "try:\n"
            "    coop.slot_map(torch.zeros(1, 1, dtype=torch.int32), None, None, None, 0, 1, 1)\n"
            "except ValueError as e:\n"
            "    print('refused:', e)\n")
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    assert "refused: paged pools are worked on by the GPU" in res.stdout


NZ = 0x1000  # a pointer that is never followed: what is refused is not launched
INVALID = -1


def _cache_of(**kw):
    d = dict(k=NZ, v=NZ, k_stride=(2048, 128, 64), v_stride=(2048, 128, 64), k_scale=None,
             v_scale=None, num_pages=4, page_size=16, heads=2, dim=64, type=0)
    d.update(kw)
    return CoopCache(*d.values())


@pytest.mark.parametrize("far", [
    dict(num_pages=(1 << 31) - 1, k_stride=(1 << 40, 128, 64)),      # 2^71 elements
    dict(num_pages=(1 << 31) - 1, v_stride=(1 << 40, 128, 64)),
    dict(num_pages=1 << 24, k_stride=(1 << 40, 128, 64)),            # wraps to a small number
    dict(page_size=(1 << 31) - 1, v_stride=(2048, 1 << 30, 64)),
    dict(num_pages=1 << 20, page_size=1 << 20, v_stride=(1 << 39, 1 << 39, 1 << 40))])
def test_pools_that_reach_past_64_bits_are_refused(far):
    """The kernels' offsets are 64-bit sums of products; where a page, a place
    and a head add up to more, the call is refused."""
    lib = coop.load_library()
    rows = CoopRows(NZ, (128, 64))
    assert lib.coop_cache_write(rows, rows, 0, NZ, 3, _cache_of(**far), None) == INVALID
    assert lib.coop_tree_attention(rows, rows, rows, 0, 4, 3, NZ, None, _cache_of(**far), NZ, 1, NZ,
                                   2, 0.125, NZ, NZ, 1 << 30, None) == INVALID


def test_rows_that_reach_past_64_bits_are_refused():
    lib = coop.load_library()
    near, far = CoopRows(NZ, (128, 64)), CoopRows(NZ, (1 << 40, 64))
    for k, v in ((near, far), (far, near)):
        assert lib.coop_cache_write(k, v, 0, NZ, 1 << 24, _cache_of(), None) == INVALID
    for q, k, v in ((far, near, near), (near, far, near), (near, near, far)):
        assert lib.coop_tree_attention(q, k, v, 0, 4, 1 << 24, NZ, None, _cache_of(), NZ, 1, NZ, 2,
                                       0.125, NZ, NZ, 1 << 50, None) == INVALID


def test_a_dimension_of_one_may_have_any_stride():
    """A single page, place or head is never stepped along (and nothing is
    launched for a call without tokens)."""
    lib = coop.load_library()
    one = _cache_of(num_pages=1, page_size=1, heads=1, k_stride=(1 << 40,) * 3, v_stride=(1 << 40,) * 3)
    rows = CoopRows(NZ, (1 << 40, 1 << 40))
    assert lib.coop_cache_write(rows, rows, 0, NZ, 0, one, None) == 0


def test_slots_that_overlap_what_is_read_are_refused():
    """Slots are written while other workgroups still read: a batch of single
    tokens has as many slots as lengths."""
    lib = coop.load_library()

    def call(slots, table=0x100000, held=0x200000, lengths=0x300000, offsets=0x400000):
        return lib.coop_slot_map(table, 64, 10, held, lengths, offsets, 64, 16, 8, slots, None)

    for name in ("table", "held", "lengths", "offsets"):
        assert call(0x500000, **{name: 0x500000}) == INVALID, name
        assert call(0x500000, **{name: 0x500000 + 63 * 8}) == INVALID, name
    assert call(0x500000, offsets=0x500000 - 64 * 8) == INVALID  # (its 65th entry)


def test_page_tables_that_overlap_one_another_are_refused():
    """The results of a call are apart from one another and from its workspace,
    and status, free pages and workspace from what is read."""
    lib = coop.load_library()
    names = ("kind", "table", "held", "lengths", "table_out", "held_out", "kind_out", "status",
             "free", "ws")

    def call(pages=8, **ptr):
        a = {**{n: 0x1000000 * (i + 1) for i, n in enumerate(names)}, **ptr}
        return lib.coop_page_tables(a["kind"], pages, a["table"], 2, 4, a["held"], a["lengths"], 16, 2,
                                    a["table_out"], a["held_out"], a["kind_out"], a["status"],
                                    a["free"], a["ws"], 1 << 16, None)

    results = ("table_out", "held_out", "kind_out", "status", "free")
    for i, x in enumerate(results):
        for y in results[:i]:
            assert call(**{x: 0x20000000, y: 0x20000000}) == INVALID, (x, y)
    for x in ("status", "free"):
        for y in names[:4]:
            assert call(**{x: 0x20000000, y: 0x20000000}) == INVALID, (x, y)
    for x in names[:-1]:
        assert call(pages=1 << 20, **{x: 0x20000000, "ws": 0x20000000}) == INVALID, x
