"""Checks of the cache entry points' host code that test_cache_host_sanitizers.py runs
in a child process with a sanitizer runtime preloaded (not collected by pytest itself).

    cache_host_checks.py LIBDLM

Sizes, frequencies, every refusal and calls with nothing to do; no GPU work is
launched.  Prints "host checks passed" at the end; any failed check raises.
"""

from __future__ import annotations

import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def main(path: str) -> None:
    from paper_2608_02625_amd import _lib as L
    L.LIB_PATH = path
    L.load(path)
    from tests import test_cache_api as T
    for name, fn in vars(T).items():
        if not name.startswith("test_"):
            continue
        marks = [m for m in getattr(fn, "pytestmark", []) if m.name == "parametrize"]
        if not marks:
            fn()
            continue
        (mark,) = marks
        keys = [k.strip() for k in mark.args[0].split(",")]
        for values in mark.args[1]:
            fn(**dict(zip(keys, values)))
    print("host checks passed")


if __name__ == "__main__":
    main(sys.argv[1])
