"""The CUDA-core form of the microscaled contractions (SAT_NO_TC=1): the same tests as the tensor-core form's, in a process of their own, since the
environment is read once.  Sizes of some thousand rows: several tiles and splits, odd widths, added to what was there, with column sums.
"""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# left out: long cases, and bounds of how the tensor-core form adds (many_terms: 132 units for 16385 terms; an FMA loop rounds each, half a unit a term)
LARGE = ("many_terms", "19001", "20000", "20001", "30000", "30001", "40000", "41001", "50001", "medium", "million")


@pytest.mark.parametrize("module,which", [
    ("test_gpu_mx.py", "product_of_4 or rows_times or weight_and_bias or empty or not_finite or far_from_one or a_4_bit_layer or captured or refus"),
    ("test_gpu_mx_edges.py", "test"),
    ("test_gpu_keep8.py", "test")], ids=["contractions", "edges", "layers"])
def test_without_tensor_cores(module, which):
    expression = f"({which}) and not ({' or '.join(LARGE)})"
    out = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-k", expression, os.path.join("tests", module)], cwd=ROOT,
                         env=dict(os.environ, SAT_NO_TC="1"), capture_output=True, text=True, timeout=600)
    assert out.returncode == 0 and " passed" in out.stdout, out.stdout[-4000:] + out.stderr[-2000:]
