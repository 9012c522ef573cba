"""Marshalling of the row operators, without a GPU: the binding needs no torch of its own."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2308_13466_b200.binding as binding
    return binding


def test_binding_without_torch(B):
    code = "import sys; sys.modules['torch'] = None\nimport paper_2308_13466_b200.binding as B\nassert B.sat_last_error is not None and len(B.EXPORTS) > 30"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)
