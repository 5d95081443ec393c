"""The host code of the calls on listed choices (listed.hip) under AddressSanitizer and UndefinedBehaviorSanitizer, on the
CPU, as test_host_sanitizer.py does for the library: a child Python drives its checks and layouts
(host_listed_checks.py).  Any sanitizer report fails the test."""
import os
import subprocess
import sys

import pytest

from test_host_sanitizer import ROOT, _build_module


def test_listed_host_code_under_sanitizers(tmp_path):
    build = _build_module()
    try:
        lib = build.build_host_sanitized(str(tmp_path))
    except FileNotFoundError as e:  # the regular build has not run in this tree
        pytest.skip(str(e))
    pre = os.environ.get("LD_PRELOAD", "")
    env = dict(os.environ, LD_PRELOAD=build.sanitizer_runtime() + (":" + pre if pre else ""), ASAN_OPTIONS="detect_leaks=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "host_listed_checks.py"), lib], env=env, capture_output=True,
                       text=True, timeout=300)
    report = r.stdout[-2000:] + r.stderr[-6000:]
    assert r.returncode == 0, report
    assert "listed checks ok" in r.stdout, report
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, report
