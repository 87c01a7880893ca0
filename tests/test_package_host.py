"""The package without torch."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_star_import_needs_no_torch():
    code = "import sys; sys.modules['torch'] = None; from paper_2607_18020_b200 import *; print(binding.__name__, build.__name__, workloads.__name__)"
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    assert done.stdout.split() == ["paper_2607_18020_b200." + m for m in ("binding", "build", "workloads")]
