"""The host side of the operators around the attention under AddressSanitizer and UndefinedBehaviorSanitizer:
the refusal and state suites of rotary positions, scores and responses run again against the sanitized build
(see test_host_sanitizers.py)."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.sanitize

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SUITES = ["tests/test_rotary.py", "tests/test_score.py", "tests/test_responses.py"]


def test_operators_under_asan_and_ubsan():
    from paper_2506_22950_amd import build

    lib = build.build_sanitized()
    env = dict(os.environ)
    env.update(INFS_LIBRARY=lib, LD_PRELOAD=build.sanitizer_runtime(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("PYTEST_XDIST_WORKER", None)
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-p", "no:xdist",
                        "-m", "not gpu", *SUITES], cwd=ROOT, env=env, capture_output=True, text=True, timeout=1200)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0, out[-6000:]
    assert " passed" in out
