"""The host code of rotary positions and of the 8-bit cache under AddressSanitizer and UndefinedBehaviorSanitizer, as
test_sanitized_host.py has it for the rest of the library.  No GPU."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = ["tests/test_fp8_host.py", "tests/test_fp8_host_edges.py"]


def _sanitized_library(hip_build) -> str:
    """The library that test_sanitized_host.py built, unless a source is newer."""
    folders = [hip_build.CSRC, os.path.join(ROOT, "include")]
    newest = max(os.path.getmtime(os.path.join(d, f)) for d in folders for f in os.listdir(d))
    if os.path.exists(hip_build.SAN_LIB) and os.path.getmtime(hip_build.SAN_LIB) > newest:
        return hip_build.SAN_LIB
    return hip_build.build_sanitized()


def test_host_code_of_the_8_bit_cache_under_address_and_ub_sanitizers():
    from paper_2507_10069_amd import build as hip_build
    try:
        runtime = hip_build.asan_runtime()
    except FileNotFoundError as e:                      # pragma: no cover
        pytest.skip(str(e))
    env = dict(os.environ)
    env["LD_PRELOAD"] = ":".join([runtime] + ([env["LD_PRELOAD"]] if env.get("LD_PRELOAD") else []))
    env["ASAN_OPTIONS"] = "detect_leaks=0:halt_on_error=1:abort_on_error=0"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    env["EMM_LIB_PATH"] = _sanitized_library(hip_build)
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "not gpu", "-p", "no:cacheprovider"] + FILES,
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    report = res.stdout[-6000:] + res.stderr[-6000:]
    if "ASan runtime does not come first" in report:    # pragma: no cover  (another preloaded library got in before it)
        pytest.skip("the sanitizer runtime cannot be preloaded first in this environment")
    assert res.returncode == 0, report
    assert "AddressSanitizer" not in report and "runtime error:" not in report, report
    assert " passed" in res.stdout
