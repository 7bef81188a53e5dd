"""The host side of the calls on caches with lengths of their own under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU, no kernel
launch): csrc/cache_api.hip with csrc/api.hip and tests/host_sanitize/cache_driver.hip, built as in test_host_sanitizers.py."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import BUILD, COMMAND, ROOT

EXE = os.path.join(BUILD, "host_cache_api_sanitized")


def test_cache_boundary_is_clean_under_asan_and_ubsan():
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    os.makedirs(BUILD, exist_ok=True)
    command = [x.replace("driver.hip", "cache_driver.hip") for x in COMMAND[:-1]] + [EXE]
    command.insert(command.index("-o"), os.path.join(ROOT, "paper_2502_04077_amd", "csrc", "cache_api.hip"))
    res = subprocess.run(command, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([EXE], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, (run.stdout + run.stderr)[-3000:]
    assert "all checks passed" in run.stdout
    assert "AddressSanitizer" not in run.stderr and "runtime error" not in run.stderr
