"""The Python forms of the binding, which are used where its extension module is not there, run the same steps."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
import pytest
sys.modules["paper_2508_11661_b200._marshal"] = None
status = pytest.main(["-x", "-q", "-p", "no:cacheprovider", "-m", "gpu",
                      "tests/test_pages_gpu.py::test_serving_steps", "tests/test_scores_gpu.py::test_other_streams",
                      "tests/test_scores_gpu.py::test_strides_and_optional_outputs", "tests/test_packed_chain_gpu.py"])
from paper_2508_11661_b200 import binding as B
assert type(B._rows).__name__ == "function"
sys.exit(int(status))
"""


def test_packed_calls_without_the_extension_module():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and " passed" in r.stdout and "skipped" not in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
