"""The package without a CUDA build of torch: it is imported, and what needs no GPU works."""
import subprocess
import sys

CODE = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2408_02897_b200 as qm
assert qm.qm_code_ld(17) == 32
assert qm.lib().qm_linear_int8(None, 0, None, None, 0, None, None, 0, 0, 1, 1, None, 0, 0, None) == 0
"""


def test_import_without_cuda_in_torch():
    r = subprocess.run([sys.executable, "-c", CODE], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
