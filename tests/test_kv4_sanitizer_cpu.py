"""The 4-bit cache's host code under AddressSanitizer and UndefinedBehaviorSanitizer, as
test_sanitizer_cpu.py runs the rest of the C ABI's."""
import os
import subprocess
import sys

from test_sanitizer_cpu import ROOT, _san_env


def test_kv4_host_tests_under_sanitizers():
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_kv4_cpu.py")],
                       env=_san_env(), capture_output=True, text=True, timeout=900, cwd=ROOT)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error:" not in r.stderr
