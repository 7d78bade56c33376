"""The host side of the paged-cache calls under AddressSanitizer (CPU only): the
refusal tests rerun in a child process that loads libfe_asan.so."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_paged_calls_under_asan():
    from paper_2509_20416_amd import build
    if not os.path.exists(build.LIB_ASAN):
        pytest.skip("libfe_asan.so not built (python -m paper_2509_20416_amd.build --asan)")
    env = dict(os.environ, LD_PRELOAD=build.asan_runtime(), FE_LIBRARY=build.LIB_ASAN,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "tests/test_paged_abi.py"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "AddressSanitizer" not in r.stderr
