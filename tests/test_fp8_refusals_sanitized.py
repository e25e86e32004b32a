"""tests/test_fp8_refusals.py again, against the host-sanitized build of the library (AddressSanitizer +
UndefinedBehaviorSanitizer on every host pass).  Any sanitizer report fails the run."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_fp8_refusals_under_address_and_undefined_behaviour_sanitizers():
    from paper_2608_27206_amd import build as b
    if not os.path.exists(b.SANITIZED_OUT):
        pytest.skip("sanitized library not built (python -m paper_2608_27206_amd.build --sanitized)")
    rt = b.sanitizer_runtime()
    env = dict(os.environ, PACE_LIB_PATH=b.SANITIZED_OUT, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    env["LD_PRELOAD"] = rt + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    code = ("import sys, pytest; from paper_2608_27206_amd import pace; "
            "assert pace.LIB_PATH.endswith('libpace_sanitized.so'); "
            "sys.exit(pytest.main(['-q', '-p', 'no:cacheprovider', 'tests/test_fp8_refusals.py']))")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert " passed" in out
