"""The argument checks and size formulas of the feed-forward entry points under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): tests/test_feedforward_host.py in a child process, on a copy of the library whose
host code is compiled with both (build.build_sanitized; errors are fatal).  The checks multiply sizes up to 2^63, so
that an overflow is what they could get wrong.  Leak detection is off: the interpreter itself keeps memory until exit.
"""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.slow
def test_feedforward_checks_pass_under_sanitizers():
    from paper_2607_01408_amd import build

    env = dict(os.environ)
    env.update({
        "LD_PRELOAD": build.sanitizer_runtime(),
        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
        "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1",
        "SPINGTP_LIBRARY": build.build_sanitized(),
    })
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_feedforward_host.py"), "-q", "-x",
                        "-p", "no:cacheprovider", "-m", "not gpu"], cwd=ROOT, env=env, capture_output=True,
                       text=True, timeout=1500)
    tail = (r.stdout + r.stderr)[-3000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
    assert " passed" in r.stdout, tail
