"""The host side of the serving operators (argument checks, the angles of a
rotation, workspace sizes) under AddressSanitizer and
UndefinedBehaviorSanitizer: their host tests run again, in a subprocess,
against the sanitized build."""

import os
import subprocess
import sys

import pytest

from test_host_sanitized import LIB, ROOT, _asan_runtime


@pytest.mark.skipif(not os.path.exists(LIB), reason="sanitized library not built (build.py --sanitize)")
def test_serving_host_code_under_asan_and_ubsan():
    rt = _asan_runtime()
    if rt is None:
        pytest.skip("no AddressSanitizer runtime for g++")
    env = dict(os.environ, DCKV_LIBRARY=LIB, LD_PRELOAD=rt,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "not gpu", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_lib_serve_host.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-3000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in tail and "runtime error" not in tail, tail
