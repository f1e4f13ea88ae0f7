"""The parts of the package that need no torch, in a process that has none."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code):
    r = subprocess.run([sys.executable, "-c", "import sys\nsys.modules['torch'] = None\n" + code], cwd=ROOT, capture_output=True,
                       text=True, timeout=100)
    assert r.returncode == 0, r.stderr
    return r.stdout


def test_estimates_and_handles_without_storage():
    out = run("""
import paper_2501_13111_amd as fp
from paper_2501_13111_amd import binding
from fpgen.workloads import CONFIGS
t, p = binding.fit_ttft_tpot([1, 3], [1.0, 2.0])
f = fp.Fingerprint(CONFIGS['tiny']['shape'], unbacked=True)
f.close()
print(t, p, hasattr(fp, 'PagedKV'))
""")
    t, p, paged = out.split()
    assert float(t) + float(p) > 0 and paged == "False"


@pytest.mark.gpu
def test_a_fingerprint():
    assert "made" in run("""
import paper_2501_13111_amd as fp
from fpgen.workloads import CONFIGS
with fp.Fingerprint(CONFIGS['tiny']['shape']) as f:
    print('made')
""")
