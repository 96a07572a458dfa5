"""The host code of window caches and drafted tokens under AddressSanitizer and
UndefinedBehaviorSanitizer, as test_sanitizer_cpu.py runs the rest of the C ABI's."""
import os
import subprocess
import sys

from test_sanitizer_cpu import ROOT, _san_env


def test_window_and_draft_host_tests_under_sanitizers():
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_window_draft_cpu.py")],
                       env=_san_env(), capture_output=True, text=True, timeout=900, cwd=ROOT)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error:" not in r.stderr
