"""The host code of sort, combine and the 8-bit products (validation, planning)
under AddressSanitizer and UndefinedBehaviorSanitizer, as
tests/test_host_sanitizers.py does it for the layer's."""
import os
import subprocess
import sys

import pytest

from paper_2609_33614_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_sort_and_fp8_abi_under_asan_and_ubsan(tmp_path):
    try:
        runtime = B.sanitizer_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    lib = str(tmp_path / "libeat_sanitized.so")
    B.build(jobs=min(8, os.cpu_count() or 1), out=lib, sanitize=True)
    env = dict(os.environ, EAT_LIB_PATH=lib, LD_PRELOAD=runtime, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", *(os.path.join(ROOT, "tests", f"test_abi_{k}.py") for k in ("sort", "fp8")),
                        "-q", "-s", "-p", "no:cacheprovider"], env=env, cwd=ROOT, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert "runtime error:" not in out and "ERROR: AddressSanitizer" not in out, out[-6000:]
    assert r.returncode == 0 and " passed" in out, out[-6000:]
