"""The host code of 8-bit pages and of chosen blocks (argument checks, launch plans, workspace sizes) under AddressSanitizer and
UndefinedBehaviorSanitizer, as the other paged calls' in test_paged_sanitizers.py."""
import os
import subprocess
import sys

import pytest

from test_paged_sanitizers import ROOT, sanitized_library


def test_host_tests_pass_under_asan_and_ubsan():
    from paper_2603_11564_amd import build
    try:
        runtime = build.asan_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    env = dict(os.environ, DAPQ_LIBRARY=sanitized_library(build), LD_PRELOAD=runtime,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",   # the interpreter itself leaks by design
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    tests = [os.path.join(ROOT, "tests", f) for f in ("test_paged_blocks_host.py", "test_paged_e4m3_host.py")]
    r = subprocess.run([sys.executable, "-m", "pytest", *tests, "-x", "-q", "-s", "-p", "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True,
                       text=True, timeout=600)
    report = r.stdout[-3000:] + r.stderr[-3000:]
    assert r.returncode == 0, report
    assert "passed" in r.stdout and "AddressSanitizer" not in report and "runtime error" not in report, report
