"""The binding loads the library with ctypes alone."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_binding_needs_neither_numpy_nor_torch():
    code = ("import sys\n"
            "sys.modules['numpy'] = sys.modules['torch'] = None\n"  # (importing them fails)
            "from paper_1802_08021_amd import sparcml as S\n"
            "assert S.lib() is not None\n"
            "assert S.workspace_size(S.OP_LOGPROB, 1, 8, 1000) > 0\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
