"""The cache entry points' host code (cache.hip) under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): everything tests/test_cache_api.py asks of the
library, in a child process that preloads the toolchain's ASan runtime."""

from __future__ import annotations

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_cache_host_paths_under_asan_and_ubsan():
    import paper_2608_02625_amd.build as b
    lib = b.build_host_sanitized()
    env = dict(os.environ, LD_PRELOAD=b.asan_runtime(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0:exitcode=23",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "cache_host_checks.py"), lib], env=env,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "host checks passed" in r.stdout, (r.returncode, r.stdout[-2000:], r.stderr[-6000:])
