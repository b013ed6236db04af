"""The argument checks, sizing and launch set-up of the cache and norm calls
under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): the tests of
test_abi_operators.py in a child process on the host-sanitized build, where any
report aborts the child."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="needs hipcc to build the sanitized host layer")
def test_operator_checks_clean_under_asan_ubsan():
    sys.path.insert(0, ROOT)
    from paper_2609_23153_amd import build as B
    env = dict(os.environ)
    env["SPARSE_ATTN_LIB"] = B.build_host_sanitized()
    env["LD_PRELOAD"] = B.asan_runtime()
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1"   # (Python's allocations look like leaks)
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_abi_operators.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert " passed" in out
