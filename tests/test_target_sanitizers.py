"""The host code of the target's operators under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): its argument tests run again in a child Python that
loads the instrumented build of the library."""

import os
import subprocess
import sys

import pytest

from test_sanitizers import LIB_ASAN, ROOT, _runtime


def test_target_checks_under_address_and_undefined_behaviour_sanitizers():
    if not os.path.exists(LIB_ASAN):
        pytest.skip("libqlin_asan.so is built by __graft_entry__.build()")
    rt = [_runtime("libasan.so"), _runtime("libubsan.so")]
    if None in rt:
        pytest.skip("g++ sanitizer runtimes not found")
    env = dict(os.environ, QLIN_LIB=LIB_ASAN, LD_PRELOAD=" ".join(rt),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-m", "not gpu",
                        os.path.join(ROOT, "tests", "test_target_abi.py")], cwd=ROOT, env=env, capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "passed" in r.stdout
