"""The checked build on the GPU: the log probabilities' parity suites pass with every
device-side bounds check compiled in (ATTT_CHECKED=1 selects libattt_checked.so), so
that no check fires on valid inputs."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SUITES = ["tests/test_gpu_logprob.py", "tests/test_gpu_logprob_heads.py", "tests/test_gpu_logprob_small_heads.py"]


def test_logprob_suites_under_the_checked_build():
    from paper_2607_03441_gb300 import build
    build.build(checked=True)
    r = subprocess.run([sys.executable, "-m", "pytest", *SUITES, "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"],
                       cwd=ROOT, env=dict(os.environ, ATTT_CHECKED="1"), capture_output=True, text=True, timeout=1200)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
