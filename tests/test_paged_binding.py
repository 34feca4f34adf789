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
