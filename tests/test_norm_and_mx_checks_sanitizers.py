"""The argument checks of the calls for normed rows and the cache in 4 bits, against the library whose host code is built with the
address and undefined-behaviour sanitizers.  Needs no GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_checks_run_clean_under_host_sanitizers(tmp_path):
    from paper_2412_12094_amd import build

    runtime = build.sanitizer_runtime()
    if not runtime:
        pytest.skip("no AddressSanitizer runtime for the host compiler")
    lib = build.build_host_sanitized(str(tmp_path / "libsepattn_san.so"))
    env = dict(os.environ, SEPATTN_LIB=lib, LD_PRELOAD=(runtime + ":" + os.environ.get("LD_PRELOAD", "")).rstrip(":"),
               ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_norm_and_mx_checks.py"), "-k", "not binding"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
