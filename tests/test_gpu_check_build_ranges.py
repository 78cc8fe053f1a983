"""The suites of magnitudes, of large pools and of rows around the numbers of CTAs against the checking build (libkvd_check.so)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


def test_the_suites_pass_on_the_checking_build():
    from paper_2603_19664_b200.build import build
    build(check=True)
    env = dict(os.environ, KVD_LIBRARY="check")
    suites = ["tests/test_gpu_cache4_ranges.py", "tests/test_gpu_pages_rounds.py", "tests/test_gpu_full_pool.py", "tests/test_gpu_sample_rows.py"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "gpu", *suites], cwd=ROOT, env=env, capture_output=True,
                       text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1500:]
