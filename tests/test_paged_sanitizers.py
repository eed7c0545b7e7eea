"""The host code of the cache in pages (argument checks, launch plans, workspace sizes) under AddressSanitizer and UndefinedBehaviorSanitizer, as the
other calls' in test_host_sanitizers.py."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def sanitized_library(build):
    """Built again where a source is newer."""
    sources = [os.path.join(build.CSRC, f) for f in os.listdir(build.CSRC)] + [os.path.join(ROOT, "include", "dapq.h"), build.__file__]
    if os.path.exists(build.SANITIZED_LIB) and os.path.getmtime(build.SANITIZED_LIB) > max(map(os.path.getmtime, sources)):
        return build.SANITIZED_LIB
    return build.build_sanitized()


def test_paged_host_tests_pass_under_asan_and_ubsan():
    from paper_2603_11564_amd import build
    try:
        runtime = build.asan_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    env = dict(os.environ, DAPQ_LIBRARY=sanitized_library(build), LD_PRELOAD=runtime,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",   # the interpreter itself leaks by design
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    tests = [os.path.join(ROOT, "tests", f) for f in ("test_paged_host.py", "test_paged_limits_host.py")]
    r = subprocess.run([sys.executable, "-m", "pytest", *tests, "-x", "-q", "-s", "-p", "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True,
                       text=True, timeout=600)
    report = r.stdout[-3000:] + r.stderr[-3000:]
    assert r.returncode == 0, report
    assert "passed" in r.stdout and "AddressSanitizer" not in report and "runtime error" not in report, report
