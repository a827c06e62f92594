"""libxpress.so is built where torch is not installed: only the binding's torch calls
need xpress_torch.so, and they say what is missing."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import importlib.abc, os, sys
class NoTorch(importlib.abc.MetaPathFinder):
    def find_spec(self, name, path=None, target=None):
        if name.split(".")[0] == "torch":
            raise ModuleNotFoundError("No module named 'torch'", name="torch")
sys.meta_path.insert(0, NoTorch())
from paper_2608_02438_gb300 import build as BLD
built = BLD.build()                     # (the test's parent has brought the library up to date)
old = BLD._stale
BLD._stale = lambda outputs, inputs: "torch" in os.path.basename(outputs[0]) or old(outputs, inputs)
assert BLD.build() == built == BLD.LIB and os.path.exists(BLD.LIB)
from paper_2608_02438_gb300 import binding as X
assert X.load().xpress_version() >= 1
"""


def test_the_library_builds_without_torch():
    from paper_2608_02438_gb300 import build as BLD
    BLD.build()
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
