"""The paged pools' binding and C refusals that need no GPU."""
import subprocess
import sys

from conftest import ROOT


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
