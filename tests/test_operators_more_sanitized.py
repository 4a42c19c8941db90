"""The CPU tests of the 4-bit operators and of queries and keys again, with the library's host code under
AddressSanitizer and UndefinedBehaviorSanitizer (validation, plans, what a call computes before its launch)."""
import os
import subprocess
import sys

import pytest

from paper_2605_25550_amd import build as B


@pytest.fixture(scope="module")
def env(tmp_path_factory):
    try:
        rt = B.sanitizer_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    lib = B.build_sanitized(str(tmp_path_factory.mktemp("asan")))
    return dict(os.environ, LD_PRELOAD=rt, DITMI_LIB=lib, ASAN_OPTIONS="detect_leaks=0",
                UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")


@pytest.mark.parametrize("name", ["test_operators_more_abi.py", "test_operators_plans.py"])
def test_host_code_under_asan_and_ubsan(env, name):
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join("tests", name), "-q", "-x", "-p", "no:cacheprovider"], cwd=B.ROOT,
                       env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
    assert " passed" in out
